"""Attention of one new token over a paged cache, and the write of its key and value, against their
definitions in 64 bits."""

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


class Setup:
    """Sequences of the given lengths in a cache whose other slots hold NaN."""

    def __init__(self, B, lens, kv, heads, dim, page, dt, order, seed=0, spread=1.0, page_gap=0, holes=0.0):
        import torch
        rng = np.random.default_rng(seed)
        self.B, self.lens, self.kv, self.heads, self.dim, self.page, self.dt, self.order = B, lens, kv, heads, dim, page, dt, order
        need = [M.ceil(n, page) for n in lens]
        self.width, pages = max(need + [1]) + 1, sum(need) + 2
        ids = rng.permutation(pages)
        self.table = np.full((len(lens), self.width), -1, np.int64)
        k = 0
        for b, m in enumerate(need):
            self.table[b, :m] = ids[k:k + m]
            k += m
        if holes:
            self.table[rng.random(self.table.shape) < holes] = -1
        rnd = M.bf16 if dt == "bf16" else (lambda a: a)
        self.keys = np.full((pages, page, kv, dim), np.nan, np.float32)
        self.values = self.keys.copy()
        for b, n in enumerate(lens):
            for t in range(n):
                p = self.table[b, t // page]
                if p >= 0:
                    self.keys[p, t % page] = rnd(rng.standard_normal((kv, dim)).astype(np.float32))
                    self.values[p, t % page] = rnd(rng.standard_normal((kv, dim)).astype(np.float32))
        self.q = rnd(rng.standard_normal((len(lens), heads, dim)).astype(np.float32) * spread)
        self.tdt = torch.bfloat16 if dt == "bf16" else torch.float32
        self.dkeys, self.dvalues = self.plane(self.keys, page_gap), self.plane(self.values, page_gap)
        self.cache = B.CacheShape.of(self.dkeys, B.HEAD_MAJOR if order == "heads" else B.SLOT_MAJOR)
        self.dtable, self.dlens = self.ints(self.table), self.ints(lens)

    def ints(self, a):
        import torch
        return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")

    def plane(self, a, gap):
        import torch
        a = a.transpose(0, 2, 1, 3) if self.order == "heads" else a
        room = torch.full((a.shape[0], a[0].size + gap), float("nan"), dtype=self.tdt, device="cuda")
        out = room[:, :a[0].size].view(a.shape[0], *a.shape[1:]) if not gap else \
            room.as_strided(a.shape, (room.stride(0), a.shape[2] * a.shape[3], a.shape[3], 1))
        out.copy_(torch.from_numpy(np.ascontiguousarray(a)))
        return out

    def feature_major(self, a):
        """[n, heads, dim] as a view of feature-major activations."""
        import torch
        n, h, d = a.shape
        return torch.from_numpy(np.ascontiguousarray(a.reshape(n, h * d).T)).to(self.tdt).cuda().view(h, d, n).permute(2, 0, 1)

    def run(self, scale, window=0, rows=None, lens=None, feature_major=False, stream=None, fill=float("nan")):
        import torch
        n = len(self.lens) if rows is None else len(rows)
        q = self.q[:n]
        qd = self.feature_major(q) if feature_major else torch.from_numpy(q).to(self.tdt).cuda()
        y = torch.full((n, self.heads, self.dim), fill, dtype=self.tdt, device="cuda")
        if feature_major:
            y = self.feature_major(np.zeros((n, self.heads, self.dim), np.float32))
        lse = torch.full((n, self.heads), fill, device="cuda")
        need = self.B.bsp_attention_workspace(self.cache, n, self.heads, self.width)
        ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        self.B.bsp_attention(self.cache, qd, self.dkeys, self.dvalues, self.dtable, self.dlens if lens is None else lens, y,
                             scale, window, None if rows is None else self.ints(rows), lse, ws, stream)
        torch.cuda.synchronize()
        return y, lse

    def check(self, y, lse, scale, window=0, rows=None, lens=None):
        """Each element: bf16 rounds every probability once (2^-8 of p |v| at most) and the output once;
        the fp32 part errs by the scores' own error, which the exponential passes on, and its sums.
        Rows also by their norm, where roundings (1.7e-3 in the mean) of many tokens add up like
        their root of squares: three times that for bf16, 1e-5 for fp32, and the scores' part."""
        y, lse = y.double().cpu().numpy(), lse.double().cpu().numpy()
        for i in range(y.shape[0]):
            r = i if rows is None else rows[i]
            ok = 0 <= r < len(self.lens)
            n = (self.lens if lens is None else lens)[r] if ok else 0
            table = self.table[r] if ok else []
            for h in range(self.heads):
                j = h // (self.heads // self.kv)
                ref, l, size, spread, qk = M.attention(self.q[i, h], self.keys[:, :, j], self.values[:, :, j], table, self.page, n,
                                               window, scale)
                if l == -np.inf:
                    assert lse[i, h] == -np.inf and (y[i, h] == 0).all()
                    continue
                score = 2 * (self.dim + 4) * M.U24 * qk
                small = 2 * score + (2 * n + 64) * M.U24
                p, u = (2.0 ** -8, 2.0 ** -8) if self.dt == "bf16" else (0.0, 2.0 ** -24)
                assert (np.abs(y[i, h] - ref) <= u * np.abs(ref) + (1 + u) * (p + small) * size).all(), (i, h)
                assert abs(lse[i, h] - l) <= score + (n + 64) * M.U24 + 4 * M.U24 * abs(l)
                norm = np.linalg.norm
                tol = 5e-3 * (norm(ref) + norm(spread)) if self.dt == "bf16" else 1e-5 * norm(ref)
                assert norm(y[i, h] - ref) <= tol + small * norm(size), (i, h)


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300]


@pytest.mark.parametrize("order", ["heads", "slots"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 80, 96, 128, 136, 192, 256])
def test_lengths_and_head_dims(B, dim, dt, order):
    s = Setup(B, LENS, 2, 6, dim, 16, dt, order, seed=dim)
    s.check(*s.run(dim ** -0.5), dim ** -0.5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kv,heads", [(1, 1), (1, 5), (1, 16), (2, 34), (3, 3), (1, 48), (4, 28), (12, 12)])
def test_head_layouts(B, kv, heads, dt):
    s = Setup(B, [5, 40, 0, 131], kv, heads, 64, 16, dt, "heads", seed=heads)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 2, 7, 16, 33, 64, 100, 256])
def test_page_sizes(B, page, dt):
    s = Setup(B, [1, 6, 7, 8, 99, 101, 257], 2, 4, 64, page, dt, "slots" if page % 2 else "heads", seed=page)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 16, 31, 100, 128, 299, 300, 5000])
def test_windows(B, window, dt):
    s = Setup(B, LENS, 2, 4, 64, 16, dt, "heads", seed=window)
    s.check(*s.run(0.125, window), 0.125, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("holes", [0.3, 0.9, 1.0])
@pytest.mark.parametrize("page", [4, 16, 64])
def test_pages_that_are_gone(B, holes, page, dt):
    """Entries that name no page, all of them too, are left out."""
    s = Setup(B, [0, 1, 40, 64, 200, 333], 2, 6, 64, page, dt, "heads", seed=page, holes=holes)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("lens,kv,heads,dim", [([5000], 1, 4, 64), ([3001, 17, 0, 1500], 2, 8, 128), ([9000, 2], 1, 1, 64),
                                               ([2049], 1, 20, 256), ([4097, 4096], 2, 2, 80)])
def test_long_sequences(B, lens, kv, heads, dim, dt):
    """Lengths that are split over workgroups and joined."""
    s = Setup(B, lens, kv, heads, dim, 16, dt, "heads", seed=sum(lens))
    s.check(*s.run(dim ** -0.5), dim ** -0.5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_many_short_sequences(B, dt):
    rng = np.random.default_rng(4)
    s = Setup(B, rng.integers(0, 50, 150).tolist(), 2, 4, 64, 16, dt, "heads", seed=3)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_sharp_softmax(B, dt):
    """Scores far apart: a maximum that comes late, after much that is then nothing."""
    s = Setup(B, [300, 1200], 1, 4, 64, 16, dt, "heads", seed=8)
    s.keys[s.table[0, 299 // 16], 299 % 16] = s.q[0, 0] * 10
    s.keys[s.table[1, 0], 0] = s.q[1, 1] * 10
    if dt == "bf16":
        s.keys = M.bf16(s.keys)
    s.dkeys = s.plane(s.keys, 0)
    s.check(*s.run(1.0), 1.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_scores_near_the_ends_of_fp32(B, dt):
    """Equal scores of great size, of either sign: the softmax is even."""
    for sign in (1.0, -1.0):
        s = Setup(B, [70], 1, 1, 64, 16, dt, "heads", seed=2)
        s.q[:] = 1.0
        s.keys[np.isfinite(s.keys)] = sign * 2.0 ** 100
        s.dkeys = s.plane(s.keys, 0)
        y, lse = s.run(1.0)
        want = s.values[s.table[0, np.arange(70) // 16], np.arange(70) % 16, 0].astype(np.float64).mean(0)
        assert np.abs(y.double().cpu().numpy()[0, 0] - want).max() < 1e-2
        assert np.isclose(float(lse[0, 0]), sign * 2.0 ** 106, rtol=1e-5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_nan_in_a_token_reaches_its_sequence_only(B, dt):
    s = Setup(B, [40, 40, 200], 2, 4, 64, 16, dt, "heads", seed=6)
    s.values[s.table[1, 0], 3, 1] = np.nan
    s.dvalues = s.plane(s.values, 0)
    y, _ = s.run(0.125)
    y = y.float().cpu().numpy()
    assert np.isnan(y[1, 2:]).all() and np.isfinite(y[1, :2]).all()
    assert np.isfinite(y[0]).all() and np.isfinite(y[2]).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["heads", "slots"])
def test_feature_major_activations_and_gaps_between_pages(B, dt, order):
    s = Setup(B, [3, 50, 129], 2, 6, 80, 16, dt, order, seed=1, page_gap=64)
    assert s.cache.page_stride == 2 * 80 * 16 + 64
    s.check(*s.run(0.1, feature_major=True), 0.1)


def test_rows_name_the_sequences(B):
    s = Setup(B, [10, 20, 300, 0, 7], 2, 4, 64, 16, "bf16", "heads", seed=5)
    rows = [2, 0, -1, 4, 5]
    s.check(*s.run(0.125, rows=rows), 0.125, rows=rows)
    rows = [4, 2]
    s.check(*s.run(0.125, rows=rows), 0.125, rows=rows)
    rows = [1, 1, 3, 2, 2]
    s.check(*s.run(0.125, rows=rows), 0.125, rows=rows)


def test_lengths_that_cannot_be(B):
    """Past the table: as long as the table.  Negative: nothing."""
    s = Setup(B, [32, 16, 40], 2, 4, 64, 16, "bf16", "heads", seed=5)
    s.table[0, 2] = s.table[0, 1]
    s.table[1, 0] = s.cache.pages + 3
    s.dtable = s.ints(s.table)
    # a whole table of pages for row 2, so that a length past it is all of them
    s.table[2] = s.table[2, 0]
    s.dtable = s.ints(s.table)
    full = s.width * 16
    y, lse = s.run(0.125, lens=s.ints([32, 16, 2 ** 31 - 1]))
    s.check(y, lse, 0.125, lens=[32, 16, full])
    y, lse = s.run(0.125, lens=s.ints([-5, 16, 10]))
    s.check(y, lse, 0.125, lens=[0, 16, 10])


def test_offsets_past_32_bits(B):
    """Pages further apart than 2^31 elements."""
    import torch
    page, kv, dim, heads = 16, 2, 64, 4
    gap = (1 << 31) + 4096
    room = torch.zeros(gap + page * kv * dim, dtype=torch.bfloat16, device="cuda")
    plane = room.as_strided((2, kv, page, dim), (gap, page * dim, dim, 1))
    cache = B.CacheShape.of(plane)
    g = torch.Generator(device="cuda").manual_seed(1)
    new = torch.randn(2, 20, kv, dim, generator=g, device="cuda").bfloat16()
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda").expand(20, 2).contiguous()
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    B.bsp_cache_append(cache, new[0], new[0], plane, plane, table, pos)
    got = torch.cat([plane[1], plane[0]], 1)[:, :20].permute(1, 0, 2)
    assert torch.equal(got, new[0])
    q = torch.randn(1, heads, dim, generator=g, device="cuda").bfloat16()
    y = torch.empty_like(q)
    ws = torch.empty(max(16, B.bsp_attention_workspace(cache, 1, heads, 2)), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([20] * 20, dtype=torch.int32, device="cuda")
    B.bsp_attention(cache, q, plane, plane, table, lens, y, 0.125, workspace=ws)
    k = new[0].double().cpu().numpy()
    for h in range(heads):
        s = k[:, h // 2] @ q[0, h].double().cpu().numpy() * 0.125
        p = np.exp(s - s.max())
        want = p @ k[:, h // 2] / p.sum()
        assert np.linalg.norm(y[0, h].double().cpu().numpy() - want) <= 5e-3 * np.linalg.norm(want)
    del room


def test_same_twice_on_streams_and_in_a_graph(B):
    """Bit for bit the same on another stream and in replays of a graph, with other work between."""
    import torch
    s = Setup(B, [700, 20, 0, 2500], 2, 8, 128, 16, "bf16", "heads", seed=12)
    first, lse1 = s.run(0.09)
    side = torch.cuda.Stream()
    second, lse2 = s.run(0.09, stream=side)
    assert torch.equal(first, second) and torch.equal(lse1, lse2)
    q = torch.from_numpy(s.q).to(s.tdt).cuda()
    y, lse = torch.empty_like(first), torch.empty_like(lse1)
    ws = torch.empty(max(16, B.bsp_attention_workspace(s.cache, 4, 8, s.width)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.bsp_attention(s.cache, q, s.dkeys, s.dvalues, s.dtable, s.dlens, y, 0.09, lse=lse, workspace=ws)
    for _ in range(4):
        y.fill_(5)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, y) and torch.equal(lse1, lse)
        s.run(0.3, window=9)


@pytest.mark.parametrize("order", ["heads", "slots"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("feature_major", [False, True])
def test_append(B, dt, order, feature_major):
    """Tokens land in their slots and nowhere else; those without a place are not written."""
    import torch
    s = Setup(B, [20, 0, 33, 50], 3, 3, 40, 16, dt, order, seed=7, page_gap=32)
    rows = [0, 0, 2, 3, 1, -1, 9, 3, 2]
    pos = [19, 3, 32, -1, 5, 2, 2, 100000, 16]
    rng = np.random.default_rng(1)
    rnd = M.bf16 if dt == "bf16" else (lambda a: a)
    k, v = (rnd(rng.standard_normal((len(rows), 3, 40)).astype(np.float32)) for _ in range(2))
    kd, vd = (s.feature_major(a) if feature_major else torch.from_numpy(a).to(s.tdt).cuda() for a in (k, v))
    B.bsp_cache_append(s.cache, kd, vd, s.dkeys, s.dvalues, s.dtable, s.ints(pos), s.ints(rows))
    for i, (r, p) in enumerate(zip(rows, pos)):
        if 0 <= r < 4 and 0 <= p < s.width * 16 and s.table[r, p // 16] >= 0:
            s.keys[s.table[r, p // 16], p % 16] = k[i]
            s.values[s.table[r, p // 16], p % 16] = v[i]
    for dev, host in ((s.dkeys, s.keys), (s.dvalues, s.values)):
        host = host.transpose(0, 2, 1, 3) if order == "heads" else host
        assert np.array_equal(dev.float().cpu().numpy(), host, equal_nan=True)


def test_append_without_rows(B):
    import torch
    s = Setup(B, [20, 7], 2, 2, 64, 16, "bf16", "heads", seed=7)
    k = torch.randn(2, 2, 64, device="cuda").bfloat16()
    B.bsp_cache_append(s.cache, k, -k, s.dkeys, s.dvalues, s.dtable, s.ints([0, 6]))
    assert torch.equal(s.dkeys[int(s.table[1, 0]), :, 6], k[1]) and torch.equal(s.dvalues[int(s.table[0, 0]), :, 0], -k[0])


def test_parts_of_one_attention_join_by_lse(B):
    """Attention over two halves, joined by their lse, is attention over both."""
    s = Setup(B, [400], 2, 4, 64, 16, "f32", "heads", seed=3)
    y, lse = s.run(0.125)
    ya, la = s.run(0.125, lens=s.ints([256]))
    yb, lb = s.run(0.125, window=400 - 256)
    f = 1 / (1 + (lb - la).exp())[..., None]
    joined = ya * f + yb * (1 - f)
    assert float((joined - y).abs().max()) < 1e-5 * float(y.abs().max())
    assert float((la.logaddexp(lb) - lse).abs().max()) < 1e-5


def test_no_sequences(B):
    import torch
    s = Setup(B, [5], 1, 1, 64, 16, "bf16", "heads")
    e = torch.empty(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    before = s.dkeys.view(torch.int16).clone()
    B.bsp_attention(s.cache, e, s.dkeys, s.dvalues, s.dtable, s.dlens, e, 1.0)
    B.bsp_cache_append(s.cache, e, e, s.dkeys, s.dvalues, s.dtable, s.ints([]))
    assert torch.equal(before, s.dkeys.view(torch.int16))
