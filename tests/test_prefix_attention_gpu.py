"""Attention of sequences that share the pages of their first tokens, against its definition in 64 bits."""

import numpy as np
import pytest

from tests import decode_model as M
from tests import sampling_model as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch   # first: the library then runs on torch's HIP runtime
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2111_11581_amd as B
    B.lib()
    return B


@pytest.fixture(autouse=True, params=["short", "long"])
def table_width(request):
    """Tables that hold no more than the sequences need, and those that could hold long ones."""
    Setup.least = 0 if request.param == "short" else 2100
    yield
    Setup.least = 0


class Setup:
    """Groups of sequences: sizes[g] members that share shared[g] tokens and have own[g][i] of their own after them
    (or, below 0, so many fewer than are shared).  Slots that hold no token are NaN.  prefix_rows: the shared pages
    belong to sequences of their own, of whose entries the members know nothing."""

    least = 0   # tokens that a table has room for

    def __init__(self, B, sizes, shared, own, kv, heads, dim, page, dt="bf16", order="heads", seed=0, spread=1.0, holes=0.0,
                 prefix_rows=False, extra=0):
        import torch
        rng = np.random.default_rng(seed)
        self.B, self.kv, self.heads, self.dim, self.page, self.dt, self.order = B, kv, heads, dim, page, dt, order
        n = sum(sizes) + extra   # the extra ones are in no group
        self.n, self.starts, self.shared = n, np.concatenate([[0], np.cumsum(sizes)]).astype(int), list(shared)
        lens = [max(0, shared[g] + own[g][i]) for g in range(len(sizes)) for i in range(sizes[g])] + [int(x) for x in rng.integers(0, 90, extra)]
        self.lens = lens + ([0] * len(sizes) if prefix_rows else [])
        self.width = max([M.ceil(x, page) for x in lens + list(shared)] + [M.ceil(self.least, page), 1]) + 1
        self.group = [g for g in range(len(sizes)) for _ in range(sizes[g])] + [None] * extra
        table, k = np.full((len(self.lens), self.width), -1, np.int64), 0
        for g, m in enumerate(sizes):
            at = list(range(self.starts[g], self.starts[g + 1]))
            whole = shared[g] // page
            part = shared[g] % page != 0
            first = np.arange(k, k + whole + part)
            k += len(first)
            for b in at:
                if not prefix_rows:
                    table[b, :len(first)] = first
                # a page that is shared in part is in the members' tables too where the tokens after it begin
                need = M.ceil(self.lens[b], page)
                new = max(0, need - whole) if prefix_rows or not part else max(0, need - whole - 1)
                begin = need - new
                table[b, begin:need] = np.arange(k, k + new)
                k += new
                if part and not prefix_rows and self.lens[b] > shared[g]:
                    table[b, whole] = first[-1]
            if prefix_rows:
                table[n + g, :len(first)] = first
        for b in range(n - extra, n):
            need = M.ceil(self.lens[b], page)
            table[b, :need] = np.arange(k, k + need)
            k += need
        self.prefix_rows = [n + g for g in range(len(sizes))] if prefix_rows else None
        pages = k + 3
        ids = rng.permutation(pages)
        self.table = np.where(table >= 0, ids[np.maximum(table, 0)], -1)
        if holes:
            self.table[rng.random(self.table.shape) < holes] = -1
        rnd = M.bf16 if dt == "bf16" else (lambda a: a)
        self.tdt = torch.bfloat16 if dt == "bf16" else torch.float32
        self.keys, self.values = (np.full((pages, page, kv, dim), np.nan, np.float32) for _ in range(2))
        for b in range(n):
            for t in {(p, s) for p, s in self.tokens(b, 0)}:
                if np.isnan(self.keys[t][0, 0]):
                    self.keys[t] = rnd(rng.standard_normal((kv, dim)).astype(np.float32))
                    self.values[t] = rnd(rng.standard_normal((kv, dim)).astype(np.float32))
        self.q = rnd(rng.standard_normal((n, heads, dim)).astype(np.float32) * spread)
        self.data = [self.plane(a) for a in (self.keys, self.values)]
        self.cache = B.CacheShape.of(self.data[0], B.HEAD_MAJOR if order == "heads" else B.SLOT_MAJOR)

    def plane(self, a):
        import torch
        return torch.from_numpy(np.ascontiguousarray(a.transpose(0, 2, 1, 3) if self.order == "heads" else a)).to(self.tdt).cuda()

    def tokens(self, b, window, lens=None, rows=None, shared=None, prefix_rows=None):
        """(page, slot) of what entry b attends to."""
        row = b if rows is None else rows[b]
        if not 0 <= row < len(self.lens):
            return []
        n = min((self.lens if lens is None else lens)[row], self.width * self.page)
        out, g = [], self.group[b]
        lead = -1
        if g is not None:
            lead = self.starts[g] if rows is None else rows[self.starts[g]]
            pr = self.prefix_rows if prefix_rows is None else prefix_rows
            lead = lead if pr is None else pr[g]
        for t in range(max(0, n - window) if window else 0, n):
            r = lead if g is not None and t < (self.shared if shared is None else shared)[g] else row
            p = self.table[r, t // self.page] if 0 <= r < len(self.lens) else -1
            if 0 <= p:
                out.append((p, t % self.page))
        return out

    def ints(self, a):
        import torch
        return None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")

    def feature_major(self, a):
        import torch
        n, h, d = a.shape
        return torch.from_numpy(np.ascontiguousarray(a.reshape(n, h * d).T)).to(self.tdt).cuda().view(h, d, n).permute(2, 0, 1)

    def run(self, scale, window=0, rows=None, lens=None, shared=None, prefix_rows=None, starts=None, feature_major=False, stream=None, lse=True):
        import torch
        q = self.feature_major(self.q) if feature_major else torch.from_numpy(self.q).to(self.tdt).cuda()
        y = self.feature_major(np.full_like(self.q, np.nan)) if feature_major else torch.full(self.q.shape, float("nan"), dtype=self.tdt, device="cuda")
        out = torch.full((self.n, self.heads), float("nan"), device="cuda") if lse else None
        g = len(self.shared) if starts is None else len(starts) - 1
        ws = torch.full((max(16, self.B.bsp_attention_prefix_workspace(self.cache, self.n, self.heads, g, self.width)),), 0xff,
                        dtype=torch.uint8, device="cuda")
        args = [self.ints(a) for a in (self.table, self.lens if lens is None else lens, self.starts if starts is None else starts,
                                       self.shared if shared is None else shared)]
        more = [self.ints(rows), self.ints(self.prefix_rows if prefix_rows is None else prefix_rows)]
        torch.cuda.synchronize()
        self.B.bsp_attention_prefix(self.cache, q, *self.data, *args, y, scale, window, *more, out, ws, stream)
        torch.cuda.synchronize()
        return y, out

    def check(self, y, lse, scale, window=0, **kw):
        """Each element: the scores' error (2 (dim + 4) roundings of sum |q k|), which the exponential passes on to
        values and sum, the sums' own (2 n roundings), probabilities cut to 16 bits for bf16, and the output's
        rounding."""
        y, lse = y.double().cpu().numpy(), lse.double().cpu().numpy()
        group = self.heads // self.kv
        for b in range(self.n):
            at = self.tokens(b, window, **kw)
            p, s = np.array(at, int).reshape(-1, 2).T
            for j in range(self.kv):
                h = slice(j * group, (j + 1) * group)
                ref, l, size, qk = S.attention(self.q[b, h], self.keys[p, s, j], self.values[p, s, j], scale)
                if not at:
                    assert (y[b, h] == 0).all() and (lse[b, h] == -np.inf).all(), b
                    continue
                n = len(at)
                score = 2 * (self.dim + 4) * S.U24 * qk[:, None]
                u, cut = (2.0 ** -8, 2.0 ** -15) if self.dt == "bf16" else (S.U24, 0.0)
                small = cut + 2 * score + (2 * n + 64) * S.U24
                assert (np.abs(y[b, h] - ref) <= u * np.abs(ref) + (1 + u) * small * size).all(), (b, j, np.abs(y[b, h] - ref).max())
                assert (np.abs(lse[b, h] - l) <= score[:, 0] + (n + 64) * S.U24 + 4 * S.U24 * np.abs(l)).all(), (b, j)


SIZES, SHARED = [1, 4, 0, 3, 2, 1], [33, 100, 5, 0, 7, 64]
OWN = [[5], [1, 40, 0, -30], [], [0, 1, 33], [9, -7], [129]]


@pytest.mark.parametrize("order", ["heads", "slots"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 80, 96, 128, 136, 192, 256])
def test_lengths_and_head_dims(B, dim, dt, order):
    s = Setup(B, SIZES, SHARED, OWN, 2, 6, dim, 16, dt, order, seed=dim, extra=2)
    s.check(*s.run(dim ** -0.5), dim ** -0.5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kv,heads", [(1, 1), (1, 5), (1, 16), (2, 34), (3, 3), (1, 48), (1, 70), (4, 28), (12, 12)])
def test_head_layouts(B, kv, heads, dt):
    s = Setup(B, SIZES, SHARED, OWN, kv, heads, 64, 16, dt, seed=heads)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 2, 7, 16, 33, 64, 100, 256])
def test_page_sizes(B, page, dt):
    s = Setup(B, SIZES, SHARED, OWN, 2, 4, 64, page, dt, "slots" if page % 2 else "heads", seed=page)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("members", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 33, 65])
def test_members(B, members, dt):
    rng = np.random.default_rng(members)
    s = Setup(B, [members, 2], [70, 50], [rng.integers(-20, 60, members), [1, 2]], 2, 8, 64, 16, dt, seed=members)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 16, 31, 50, 99, 100, 141, 1000])
def test_windows(B, window, dt):
    s = Setup(B, SIZES, SHARED, OWN, 2, 6, 80, 7, dt, seed=window)
    s.check(*s.run(0.11, window), 0.11, window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pages_that_hold_nothing(B, dt):
    for seed, holes in ((0, 0.3), (1, 0.7), (2, 1.0)):
        s = Setup(B, SIZES, SHARED, OWN, 2, 6, 64, 7, dt, "slots", seed=seed, holes=holes)
        s.check(*s.run(0.125), 0.125)
    s = Setup(B, SIZES, SHARED, OWN, 2, 6, 64, 7, dt, seed=3)
    s.table[s.table == s.table[1, 2]] = 10 ** 6   # past the cache
    keep = s.table.copy()
    y, lse = s.run(0.125)
    s.table = np.where(keep == 10 ** 6, -1, keep)
    s.check(y, lse, 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_shared_pages_of_another_sequence(B, dt):
    s = Setup(B, SIZES, SHARED, OWN, 2, 6, 64, 16, dt, seed=4, prefix_rows=True, extra=3)
    s.check(*s.run(0.125), 0.125)
    for rows in ([-1, 10 ** 6, 3, 4, len(s.lens), 0], [s.prefix_rows[1]] * 6):
        s2 = Setup(B, SIZES, SHARED, OWN, 2, 6, 64, 16, dt, seed=4, prefix_rows=True, extra=3)
        s2.prefix_rows = rows
        # what members now attend to may be slots that were never written
        s2.keys, s2.values = np.nan_to_num(s2.keys, nan=0.25), np.nan_to_num(s2.values, nan=0.5)
        s2.data = [s2.plane(a) for a in (s2.keys, s2.values)]
        s2.check(*s2.run(0.125), 0.125)


def test_rows_in_any_order_and_out_of_range(B):
    s = Setup(B, [3, 4], [40, 64], [[1, 2, 3], [5, 6, 7, 8]], 2, 6, 64, 16, seed=5)
    rows = [1, 0, -1, 5, 6, 10 ** 6, 3]
    s.check(*s.run(0.125, rows=rows), 0.125, rows=rows)
    rows = [-1, 0, 1, 7, 4, 5, 6]   # the first of each group is none: nothing is shared with the others
    s.check(*s.run(0.125, rows=rows), 0.125, rows=rows)
    s.check(*s.run(0.125, rows=[0] * 7), 0.125, rows=[0] * 7)


def test_lengths_and_shared_tokens_out_of_range(B):
    s = Setup(B, SIZES, SHARED, OWN, 2, 6, 64, 16, "f32", seed=6)
    lens = [10 ** 9, -5, 2 ** 31 - 1, 3, 50, 0, -2 ** 31, 1, 2, 90, 91]
    s.keys, s.values = np.nan_to_num(s.keys, nan=0.25), np.nan_to_num(s.values, nan=0.5)
    s.data = [s.plane(a) for a in (s.keys, s.values)]
    for shared in (s.shared, [10 ** 9, -3, 2 ** 31 - 1, 10 ** 6, 40, -2 ** 31]):
        s.check(*s.run(0.125, lens=lens, shared=shared), 0.125, lens=lens, shared=shared)


def test_groups_in_part_of_the_batch(B):
    s = Setup(B, [3, 4], [40, 64], [[1, 2, 3], [5, 6, 7, 8]], 2, 6, 64, 16, seed=7)
    whole = s.run(0.125)
    for starts, shared in (([0], []), ([2, 2, 2], [9, 9]), ([1, 3, 7], [40, 64]), ([0, 3, 5], [40, 64]), ([3, 7], [64]), ([7, 7], [3])):
        y, lse = s.run(0.125, starts=starts, shared=shared)
        s.check(y, lse, 0.125)   # tables agree, so that it does not matter what is said to be shared
    assert whole[0].shape == (7, 6, 64)


def test_starts_that_make_no_sense_stay_within_bounds(B):
    """Nothing is promised of the values, but every output is written (0 and -Inf where there are no tokens)."""
    import torch
    s = Setup(B, [3, 4], [40, 64], [[1, 2, 3], [5, 6, 7, 8]], 2, 6, 64, 16, seed=8)
    s.data = [s.plane(np.nan_to_num(a, nan=0.25)) for a in (s.keys, s.values)]
    for starts in ([5, 2, 9], [-4, 3, 100], [2 ** 31 - 1, -2 ** 31, 3], [7, 0, 7], [-5, -3, -1], [100, 200, 300]):
        y, lse = s.run(0.125, starts=starts)
        assert not y.isnan().any() and not lse.isnan().any()


@pytest.mark.parametrize("dt,order", [("bf16", "heads"), ("bf16", "slots"), ("f32", "heads")])
def test_long_prefix(B, dt, order):
    rng = np.random.default_rng(9)
    s = Setup(B, [5, 1, 20], [5000, 300, 2311], [rng.integers(-3000, 100, 5), [3], rng.integers(1, 200, 20)], 2, 8, 128, 16, dt, order, seed=9, extra=4)
    s.check(*s.run(0.088), 0.088)
    s.check(*s.run(0.088, feature_major=True), 0.088)
    s.check(*s.run(0.088, 1500), 0.088, 1500)


def test_one_long_prefix_few_heads(B):
    s = Setup(B, [2], [20011], [[1, 300]], 1, 1, 64, 64, "bf16", seed=10)
    s.check(*s.run(0.125), 0.125)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 72, 128, 256])
def test_column_blocks(B, dim, dt):
    """Groups of every number of columns that is worked on in another way, over several stages and tiles."""
    rng = np.random.default_rng(dim)
    sizes = [1, 4, 8, 9, 16, 17, 32, 33, 64, 71, 100]
    shared = [int(x) for x in rng.integers(900, 2300, len(sizes))]
    s = Setup(B, sizes, shared, [rng.integers(0, 150, m) for m in sizes], 1, 4, dim, 16, dt, "slots" if dim == 72 else "heads", seed=dim, holes=0.02)
    s.check(*s.run(dim ** -0.5), dim ** -0.5)
    s.check(*s.run(dim ** -0.5, feature_major=True, window=1500), dim ** -0.5, 1500)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kv,heads,dim,members", [(3, 6, 64, 60), (8, 8, 64, 40), (5, 100, 40, 30), (6, 18, 128, 70), (8, 16, 136, 20)])
def test_short_ends_of_many_sequences(B, kv, heads, dim, members, dt):
    """Several key heads of a sequence's own tokens are worked on together, not always as many as there is room for."""
    rng = np.random.default_rng(kv)
    own = [rng.integers(0, 200, members), rng.integers(-50, 300, 3)]
    s = Setup(B, [members, 3], [130, 60], own, kv, heads, dim, 16, dt, seed=kv, extra=2)
    s.check(*s.run(dim ** -0.5), dim ** -0.5)


@pytest.mark.parametrize("dt,page,order,batch,kv,heads,dim,longest", [
    ("bf16", 64, "heads", 64, 8, 64, 128, 12000), ("bf16", 16, "slots", 40, 8, 32, 64, 9000), ("bf16", 7, "heads", 33, 4, 16, 96, 6000),
    ("f32", 16, "heads", 24, 8, 32, 128, 4000), ("bf16", 64, "heads", 12, 4, 16, 256, 5000)])
def test_as_attention_over_long_prefixes(B, dt, page, order, batch, kv, heads, dim, longest):
    """Tasks over several tiles of tokens, against attention that shares nothing (which has tests of its own)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(batch)
    tdt = torch.bfloat16 if dt == "bf16" else torch.float32
    groups = 3
    starts = [0, batch // 2, batch // 2 + 1, batch]
    whole = [longest // page, longest // (3 * page), longest // (2 * page)]   # shared pages
    own = torch.randint(0, 40, (batch,), generator=torch.Generator().manual_seed(1)).tolist()
    rows, used = [], 0
    for g in range(groups):
        first = list(range(used, used + whole[g]))
        used += whole[g]
        for b in range(starts[g], starts[g + 1]):
            n = M.ceil(own[b], page)
            rows.append(first + list(range(used, used + n)))
            used += n
    lens = [whole[g] * page + own[b] for g in range(groups) for b in range(starts[g], starts[g + 1])]
    width = max(map(len, rows)) + 1
    ids = torch.randperm(used + 1, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    for b, r in enumerate(rows):
        table[b, :len(r)] = ids[torch.tensor(r, device="cuda", dtype=torch.long)]
    inner = (kv, page) if order == "heads" else (page, kv)
    data = [torch.randn(used + 1, *inner, dim, generator=gen, device="cuda").to(tdt) for _ in range(2)]
    cache = B.CacheShape.of(data[0], B.HEAD_MAJOR if order == "heads" else B.SLOT_MAJOR)
    q = torch.randn(batch, heads, dim, generator=gen, device="cuda").to(tdt)

    def ints(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")
    y, z = torch.empty_like(q), torch.empty_like(q)
    lse, lse2 = (torch.empty(batch, heads, device="cuda") for _ in range(2))
    ws = torch.full((B.bsp_attention_prefix_workspace(cache, batch, heads, groups, width) + 16,), 0xff, dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(B.bsp_attention_workspace(cache, batch, heads, width) + 16, dtype=torch.uint8, device="cuda")
    for window in (0, longest - 100):
        for scale in (dim ** -0.5, 0.5):
            B.bsp_attention_prefix(cache, q, *data, table, ints(lens), ints(starts), ints([n * page for n in whole]), y, scale, window,
                                   None, None, lse, ws)
            B.bsp_attention(cache, q, *data, table, ints(lens), z, scale, window, None, lse2, ws2)
            torch.cuda.synchronize()
            # Each within its bounds of the same values: the output's rounding; scores of up to some 4 sqrt(dim) units, whose 2 (dim + 4)
            # roundings the exponential passes on; and the sums' own, over up to 12000 tokens.
            u = 2.0 ** -8 if dt == "bf16" else S.U24
            score = 2 * (dim + 4) * S.U24 * scale * dim
            size = (2 * score + (2 * longest + 64) * S.U24 + (2.0 ** -15 if dt == "bf16" else 0)) * 5
            assert ((y.double() - z.double()).abs() <= 2 * u * z.double().abs() + 2 * size).all()
            assert ((lse.double() - lse2.double()).abs() <= 2 * (score + (longest + 64) * S.U24) + 8 * S.U24 * lse.double().abs()).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_what_one_member_attends_to_does_not_reach_another(B, dt):
    """NaN and Inf in tokens past the end, or before the window, of some members of a group."""
    import torch
    for seed, (m, group) in enumerate(((3, 2), (24, 4), (70, 4))):
        rng = np.random.default_rng(seed)
        s = Setup(B, [m], [1300], [[100, 40] + list(rng.integers(-900, 100, m - 2))], 1, group, 64, 16, dt, seed=seed)
        for window in (0, 1150):
            longest = s.run(0.125, window)[0]
            bad = sorted((n - (window or n), n) for n in s.lens)
            assert bad[0] != bad[-1]
            for at, value in ((s.lens[0] - 1, float("nan")), (1250, float("inf")), (1299, float("nan")), (160, float("nan"))):
                keys, values = s.keys.copy(), s.values.copy()
                page, slot = s.table[0, at // 16], at % 16
                keys[page, slot] = value
                values[page, slot] = value
                t = Setup.__new__(Setup)
                t.__dict__.update(s.__dict__)
                t.data = [t.plane(a) for a in (keys, values)]
                y, lse = t.run(0.125, window)
                for b in range(s.n):
                    if (page, slot) not in s.tokens(b, window):
                        assert torch.equal(y[b], longest[b]) or (y[b].isfinite().all() and lse[b].isfinite().all() or s.lens[b] == 0), (b, at)


def test_scores_far_apart(B):
    """Probabilities from 1 to nothing; maxima that grow from step to step."""
    for dt in ("bf16", "f32"):
        s = Setup(B, [4, 6], [700, 65], [[1, 2, 3, 4]] + [[30] * 6], 2, 4, 64, 16, dt, seed=11, spread=30.0)
        s.check(*s.run(0.5), 0.5)
        at = np.argsort(np.arange(len(s.keys)))
        s.keys *= (1 + at)[:, None, None, None] / len(at) * 2
        if dt == "bf16":
            s.keys = M.bf16(s.keys)
        s.data[0] = s.plane(s.keys)
        s.check(*s.run(0.5), 0.5)
        s.check(*s.run(0.0), 0.0)
        s.check(*s.run(-0.5), -0.5)


def test_as_attention_without_groups(B):
    import torch
    s = Setup(B, [6, 5], [200, 333], [[1, 9, 40, 2, 0, -100], [5] * 5], 2, 8, 128, 16, seed=12)
    y, lse = s.run(0.088)
    z, lse2 = torch.empty_like(y), torch.empty_like(lse)
    ws = torch.empty(max(16, B.bsp_attention_workspace(s.cache, s.n, s.heads, s.width)), dtype=torch.uint8, device="cuda")
    B.bsp_attention(s.cache, torch.from_numpy(s.q).to(s.tdt).cuda(), *s.data, s.ints(s.table), s.ints(s.lens), z, 0.088, 0, None, lse2, ws)
    torch.cuda.synchronize()
    # both are within their bounds of the same values: one output step of each
    assert ((y.double() - z.double()).abs() <= 2.0 ** -7 * z.double().abs() + 1e-4).all() and torch.allclose(lse, lse2, atol=1e-5)


def test_many_sequences(B):
    rng = np.random.default_rng(13)
    s = Setup(B, [10] * 100, rng.integers(0, 40, 100), [rng.integers(0, 20, 10) for _ in range(100)], 1, 2, 64, 16, seed=13, extra=24)
    assert s.n == 1024
    s.check(*s.run(0.125), 0.125)
    s = Setup(B, [1] * 300, rng.integers(0, 70, 300), [[int(x)] for x in rng.integers(0, 20, 300)], 1, 2, 64, 16, "f32", seed=14)
    s.check(*s.run(0.125), 0.125)
    s = Setup(B, [700], [90], [rng.integers(-80, 20, 700)], 1, 1, 64, 16, "bf16", seed=15)
    s.check(*s.run(0.125), 0.125)


def test_results_do_not_change_from_run_to_run(B):
    import torch
    rng = np.random.default_rng(16)
    s = Setup(B, [20, 3], [3000, 900], [rng.integers(1, 200, 20), [1, 2, 3]], 2, 8, 128, 16, seed=16)
    y, lse = s.run(0.088)
    for _ in range(5):
        z, lse2 = s.run(0.088)
        assert torch.equal(y, z) and torch.equal(lse, lse2)
    z, _ = s.run(0.088, lse=False)
    assert torch.equal(y, z)


def test_streams_and_graphs(B):
    import torch
    rng = np.random.default_rng(17)
    s = Setup(B, [20, 3], [1000, 300], [rng.integers(1, 100, 20), [1, 2, 3]], 2, 8, 64, 16, seed=17)
    s.check(*s.run(0.125, stream=torch.cuda.Stream()), 0.125)
    q = torch.from_numpy(s.q).to(s.tdt).cuda()
    dev = [s.ints(a) for a in (s.table, s.lens, s.starts, s.shared)]
    need = max(16, B.bsp_attention_prefix_workspace(s.cache, s.n, s.heads, 2, s.width))
    graphs, outs, spaces = [], [], []
    for _ in range(2):
        outs.append((torch.empty_like(q), torch.empty(s.n, s.heads, device="cuda")))
        spaces.append(torch.full((need,), 0xff, dtype=torch.uint8, device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.bsp_attention_prefix(s.cache, q, *s.data, *dev, outs[-1][0], 0.125, 0, None, None, outs[-1][1], spaces[-1])
    lens = list(s.lens)
    for turn in range(4):
        dev[1].copy_(s.ints(lens))
        for y, lse in outs:
            y.fill_(float("nan")), lse.fill_(float("nan"))
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        s.check(*outs[turn % 2], 0.125, lens=lens)
        lens = [max(0, n - int(rng.integers(0, 400))) for n in s.lens]
        s.run(0.125)   # eager work in between


def test_an_offset_past_32_bits(B):
    """Pages 2^31 elements into the cache."""
    import torch
    page, kv, dim = 64, 8, 128
    pages = (1 << 31) // (page * kv * dim) + 4
    keys, values = (torch.empty(pages, kv, page, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(18)
    s = Setup(B, [3], [128], [[1, 30, 64]], kv, kv, dim, page, seed=18)
    assert len(s.keys) <= 8 and s.table.max() < len(s.keys)
    to = np.array([pages - 1 - i if i < 4 else i - 4 for i in range(8)])
    for i in range(len(s.keys)):
        keys[int(to[i])], values[int(to[i])] = s.data[0][i], s.data[1][i]
    s.table = np.where(s.table >= 0, to[np.maximum(s.table, 0)], -1)
    s.data, s.cache = [keys, values], B.CacheShape.of(keys)
    y, lse = s.run(0.088)
    back = {int(p): i for i, p in enumerate(to)}
    s.table = np.array([[back.get(int(e), -1) for e in row] for row in s.table])
    s.check(y, lse, 0.088)


def test_units_that_do_not_fill_their_tasks(B):
    """Nine key heads go eight to a task, and most tasks in two pieces: no more than the workspace has room for."""
    import torch
    n = 257
    s = Setup(B, [1] * n, [1] * (n - 1) + [3200], [[200]] * n, 9, 9, 8, 16, seed=11)
    need = B.bsp_attention_prefix_workspace(s.cache, n, 9, n, s.width)
    ws = torch.full((need + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    q, y = torch.from_numpy(s.q).to(s.tdt).cuda(), torch.full(s.q.shape, float("nan"), dtype=s.tdt, device="cuda")
    out = torch.empty(n, 9, device="cuda")
    B.bsp_attention_prefix(s.cache, q, *s.data, s.ints(s.table), s.ints(s.lens), s.ints(s.starts), s.ints(s.shared), y, 0.35, 0, None, None,
                           out, ws[:need])
    torch.cuda.synchronize()
    s.check(y, out, 0.35)
    assert bool((ws[need:] == 0xff).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_more_workgroups_than_fill_the_card(B, dim, dt):
    rng = np.random.default_rng(dim)
    s = Setup(B, [100, 30], [50, 33], [rng.integers(-20, 20, 100), rng.integers(0, 9, 30)], 2, 6, dim, 16, dt, seed=dim)
    s.check(*s.run(dim ** -0.5), dim ** -0.5)
