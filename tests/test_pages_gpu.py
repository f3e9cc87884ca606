"""Care of a paged cache against a model of it in plain Python: tables, lengths, counts, the pages
given out, and what every slot holds, are equal."""

import numpy as np
import pytest

from tests import decode_model as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch   # first: the library then runs on torch's HIP runtime
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2111_11581_amd as B
    B.lib()
    return B


class Device:
    """The same state on the device; a slot holds its token's number in every element, plus its plane's."""

    def __init__(self, B, seqs, width, pages, page, planes=3, kv=2, dim=8, dt="f32", order="heads", n=64, gap=0):
        import torch
        self.B, self.model = B, M.Pages(seqs, width, pages, page)
        self.planes, self.order, self.page, self.kv, self.dim = planes, order, page, kv, dim
        tdt = torch.float32 if dt == "f32" else torch.bfloat16
        inner = (kv, page) if order == "heads" else (page, kv)
        room = torch.zeros(planes, pages, page * kv * dim + gap, dtype=tdt, device="cuda")
        self.data = room.as_strided((planes, pages, *inner, dim), (*room.stride()[:2], inner[1] * dim, dim, 1))
        self.cache = B.CacheShape.of(self.data[0], B.HEAD_MAJOR if order == "heads" else B.SLOT_MAJOR)
        self.table, self.lens, self.refs = self.ints(self.model.table), self.ints(self.model.lens), self.ints(self.model.refs)
        self.scratch = torch.full((B.bsp_cache_scratch(self.cache, seqs, width, n),), 0x5A, dtype=torch.uint8, device="cuda")

    def ints(self, a):
        import torch
        return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")

    def fork(self, parents, children):
        self.model.fork(parents, children)
        self.B.bsp_cache_fork(self.table, self.lens, self.refs, self.ints(parents), self.ints(children), self.scratch)

    def release(self, rows):
        self.model.release(rows)
        self.B.bsp_cache_release(self.table, self.lens, self.refs, self.ints(rows))

    def extend(self, rows, counts, first_token=None):
        """And writes the new tokens, numbered on from first_token."""
        import torch
        want = self.model.extend(rows, counts)
        pos = self.ints([-77] * len(rows))
        self.B.bsp_cache_extend(self.cache, self.data, self.table, self.lens, self.refs, self.ints(rows), self.ints(counts),
                                pos, self.scratch)
        assert pos.tolist() == want
        if first_token is None:
            return want
        tokens = [(r, p + j) for r, p, c in zip(rows, want, counts) for j in range(c) if p >= 0]
        if tokens:
            ids = np.arange(len(tokens)) + first_token
            for (r, p), t in zip(tokens, ids):
                self.model.write(r, p, t)
            kv = torch.tensor(ids, dtype=self.data.dtype, device="cuda")[:, None, None].expand(-1, self.kv, self.dim)
            rr, pp = self.ints([r for r, _ in tokens]), self.ints([p for _, p in tokens])
            for plane in range(0, self.planes - 1, 2):
                self.B.bsp_cache_append(self.cache, kv + plane, kv + plane + 1, self.data[plane], self.data[plane + 1],
                                        self.table, pp, rr)
            if self.planes % 2:
                last = self.data[self.planes - 1]
                self.B.bsp_cache_append(self.cache, kv + self.planes - 1, kv + self.planes - 1, last, last, self.table, pp, rr)
        return want

    def compact(self):
        info = self.ints([-1, -1])
        self.B.bsp_cache_compact(self.cache, self.data, self.table, self.refs, info, self.scratch)
        assert tuple(info.tolist()) == self.model.compact()

    def check(self):
        assert np.array_equal(self.table.cpu().numpy(), self.model.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.model.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.model.refs)
        want = self.model.data[None, :, None, :, None] if self.order == "heads" else self.model.data[None, :, :, None, None]
        got = self.data.double().cpu().numpy()
        for plane in range(self.planes):
            w = np.where(want[0] > 0, want[0] + plane, 0)
            assert np.array_equal(got[plane], np.broadcast_to(w, got[plane].shape)), plane


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("page", [1, 4, 7])
def test_random_lives(B, page, seed):
    """Sequences begin, grow, fork, end and move, until the pages run out and after."""
    rng = np.random.default_rng(seed * 10 + page)
    d = Device(B, 9, 12, 60, page, planes=3 + seed % 2, order=["heads", "slots"][seed % 2], gap=16 * (seed % 3))
    token = 1
    for step in range(40):
        op = rng.choice(["extend", "extend", "extend", "fork", "release", "compact"])
        rows = rng.permutation(9)[:rng.integers(1, 7)].tolist()
        if op == "extend":
            counts = rng.integers(0, 3 * page + 2, len(rows)).tolist()
            d.extend(rows, counts, token)
            token += sum(counts)
        elif op == "fork":
            parents = rng.integers(0, 9, len(rows)).tolist()
            d.fork(parents, rows)
        elif op == "release":
            d.release(rows[:2])
        else:
            d.compact()
        if step % 5 == 4:
            d.check()
    d.check()


def test_beams_permuted_in_place(B):
    """Children that are parents of others at once."""
    d = Device(B, 4, 8, 40, 4)
    d.extend([0, 1, 2, 3], [5, 9, 3, 8], 1)
    d.fork([1, 0, 0, 3], [0, 1, 2, 3])
    d.check()
    d.extend([0, 1, 2, 3], [1, 1, 1, 1], 100)
    d.check()


def test_all_or_nothing(B):
    d = Device(B, 3, 4, 6, 4)
    assert d.extend([0, 1], [8, 8], 1) == [0, 0]
    assert d.extend([0, 1, 2], [1, 4, 9], 50) == [-1, -1, -1]   # one page more than there are
    d.check()
    assert d.extend([0, 1], [1, 4], 80) == [8, 8]
    assert d.extend([2], [0]) == [0]
    assert d.extend([2], [1]) == [-1]
    d.check()
    d.release([0])
    assert d.extend([2], [17]) == [-1]   # wider than the table
    d.check()


def test_shared_last_page_is_copied_for_each(B):
    d = Device(B, 6, 4, 30, 8, order="slots")
    d.extend([0], [13], 1)
    d.fork([0] * 5, [1, 2, 3, 4, 5])
    d.check()
    d.extend([1, 2, 0, 5], [1, 2, 1, 4], 40)
    d.check()
    assert d.refs.max() == 6
    d.extend([3, 4], [1, 1], 80)
    d.check()


def test_a_last_entry_that_names_no_page_gets_one(B):
    d = Device(B, 2, 4, 10, 4)
    d.extend([0], [6], 1)
    d.model.drop([d.model.table[0, 1]])
    d.model.table[0, 1] = -1
    d.table, d.refs = d.ints(d.model.table), d.ints(d.model.refs)
    d.model.data[1] = 0
    d.data[:, 1] = 0
    d.extend([0], [1], 20)
    d.check()


def test_rows_out_of_range_are_left_out(B):
    d = Device(B, 3, 4, 20, 4)
    assert d.extend([1, -1, 7], [5, 5, 5], 1) == [0, -1, -1]
    d.fork([1, 5, 1, -3], [0, 2, 3, 0])
    d.release([-1, 3, 1])
    d.check()


@pytest.mark.parametrize("n", [1, 700, 2500])
def test_many_sequences(B, n):
    """More sequences than one pass of the plan takes, and pages in any order."""
    d = Device(B, n, 3, 3 * n + 50, 2, planes=1, kv=1, n=n)
    rng = np.random.default_rng(n)
    d.extend(list(range(n)), rng.integers(0, 4, n).tolist(), 1)
    d.fork(rng.integers(0, n, n).tolist(), list(range(n)))
    d.extend(rng.permutation(n).tolist(), rng.integers(0, 2, n).tolist(), 20000)
    d.check()
    d.release(rng.permutation(n)[: n // 2].tolist())
    d.compact()
    d.check()


def test_compact_moves_the_fewest_pages(B):
    d = Device(B, 8, 6, 5000, 4, dt="bf16", dim=16)
    d.extend(list(range(8)), [24] * 8, 1)
    d.release([0, 3, 4])
    before = d.table.clone()
    d.compact()
    d.check()
    moved = (before != d.table).sum()
    assert moved == 18   # of the 30 live pages 6 .. 17 and 30 .. 47, those past the first 30
    d.compact()
    d.check()


def test_compact_empty_and_full(B):
    d = Device(B, 4, 4, 16, 4)
    d.compact()
    d.check()
    d.extend([0, 1, 2, 3], [16] * 4, 1)
    d.compact()
    d.check()


@pytest.mark.parametrize("dt,order", [("f32", "heads"), ("bf16", "slots")])
def test_copy(B, dt, order):
    d = Device(B, 1, 1, 12, 5, planes=4, dt=dt, order=order, gap=8)
    d.data.copy_(d.data.new_tensor(np.random.default_rng(0).integers(0, 200, d.data.shape)))
    want = d.data.clone()
    for a, b in ((3, 0), (7, 11), (3, 4)):
        want[:, b] = want[:, a]
    d.B.bsp_cache_copy(d.cache, d.data, d.ints([3, 7, 12, 3, 1]), d.ints([0, 11, 1, 4, -1]))
    assert (d.data == want).all()
    d.B.bsp_cache_copy(d.cache, d.data, d.ints([]), d.ints([]))


def test_a_step_of_a_beam_search_in_a_graph(B):
    """Fork, extend and append replayed with other state in the tables each time."""
    import torch
    d = Device(B, 8, 6, 64, 4)
    d.extend([0, 1], [6, 9], 1)
    parents, children, counts = d.ints([0, 0, 1, 1]), d.ints([2, 3, 4, 5]), d.ints([1, 1, 1, 1])
    pos = d.ints([0] * 4)
    kv = torch.full((4, 2, 8), 500.0, device="cuda")

    def step():
        B.bsp_cache_fork(d.table, d.lens, d.refs, parents, children, d.scratch)
        B.bsp_cache_extend(d.cache, d.data, d.table, d.lens, d.refs, children, counts, pos, d.scratch)
        B.bsp_cache_append(d.cache, kv, kv + 1, d.data[0], d.data[1], d.table, pos, children)

    keep = [t.clone() for t in (d.table, d.lens, d.refs, d.data)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    eager = [t.clone() for t in (d.table, d.lens, d.refs, d.data, pos)]
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t, k in zip((d.table, d.lens, d.refs, d.data), keep):
            t.copy_(k)
        pos.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip((d.table, d.lens, d.refs, d.data, pos), eager):
            assert torch.equal(t, e)


@pytest.mark.parametrize("page", [1, 4])
def test_more_tokens_than_numbers(B, page):
    """Counts whose sum with the length passes 32 bits."""
    d = Device(B, 3, 4, 20, page)
    d.extend([0], [3], 1)
    assert d.extend([1, 0], [1, 2**31 - 1]) == [-1, -1]
    assert d.extend([1, 2], [2**31 - 1] * 2) == [-1, -1]
    d.check()


@pytest.mark.parametrize("dt,order", [("f32", "slots"), ("bf16", "heads")])
def test_pages_of_several_chunks(B, dt, order):
    """Pages of more than 32 KB, whose copies are cut."""
    d = Device(B, 6, 2, 9, 150, planes=3, kv=3, dim=104, dt=dt, order=order, gap=8)
    d.extend([3, 0], [50, 201], 1)   # numbers up to 253 are exact in bf16 too
    d.fork([0, 0], [1, 2])
    d.extend([1, 2, 0], [0, 2, 1])
    d.release([3])
    d.compact()
    d.check()
