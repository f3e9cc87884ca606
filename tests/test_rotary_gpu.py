"""Rotary positions with norms of heads, alone and on the way into the cache, against their definition
in 64 bits."""

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


def tdt(dt):
    import torch
    return torch.bfloat16 if dt == "bf16" else torch.float32


def draw(rng, shape, dt):
    a = rng.standard_normal(shape).astype(np.float32)
    return M.bf16(a) if dt == "bf16" else a


def place(a, dt, layout):
    """[n, heads, dim] on the device: token by token, feature-major, heads outside, or with gaps everywhere."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).to(tdt(dt)).cuda()
    n, h, d = t.shape
    if layout == "features":
        return t.permute(1, 2, 0).contiguous().permute(2, 0, 1)
    if layout == "heads":
        return t.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    if layout == "gaps":
        room = torch.full((n + 1, h + 2, 2 * d + 3), 7.0, dtype=t.dtype, device="cuda")
        out = room[1:, 1:h + 1, 1:1 + 2 * d:2]
        out.copy_(t)
        return out
    if layout == "wide":   # rows with a gap that keeps them at 16 bytes
        room = torch.full((n, h + 1, d + 16), 7.0, dtype=t.dtype, device="cuda")
        out = room[:, :h, :d]
        out.copy_(t)
        return out
    if layout == "odd":    # rows that begin anywhere
        room = torch.full((n, h * d + 1), 7.0, dtype=t.dtype, device="cuda")
        out = room[:, 1:].unflatten(1, (h, d))
        out.copy_(t)
        return out
    return t


def ints(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def close(got, want, bound, dt):
    got = got.double().cpu().numpy()
    u = 2.0 ** -8 if dt == "bf16" else S.U24
    assert (np.abs(got - want) <= u * np.abs(want) + (1 + u) * bound).all(), np.abs(got - want).max()


def run(B, x, pos, dims, dt, interleaved=False, factor=1.0, norm=None, eps=1e-5, layout="tokens", out="tokens", freq=None,
        inplace=False, stream=None):
    import torch
    freq = S.freqs(dims, 10000.0) if freq is None else freq
    xd = place(x, dt, layout)
    yd = xd if inplace else place(np.full_like(x, np.nan), dt, out)
    rope = B.Rope(B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, dims, factor)
    fd = torch.tensor(freq, dtype=torch.float64, device="cuda") if dims else None
    nd = None if norm is None else torch.from_numpy(norm).cuda()
    torch.cuda.synchronize()
    B.bsp_rotary(B.BF16 if dt == "bf16" else B.F32, rope, fd, xd, ints(pos), yd, nd, eps, stream)
    torch.cuda.synchronize()
    want, bound = S.rotate(x, pos, freq, interleaved, np.float32(factor).astype(np.float64), norm, eps)
    close(yd, want, bound, dt)
    if norm is None:   # what is passed on is passed on as it is
        assert (yd[:, :, dims:].float().cpu().numpy() == x[:, :, dims:]).all()
    return yd


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,dims", [(64, 64), (128, 128), (256, 256), (256, 64), (80, 80), (80, 40), (96, 32), (128, 30), (72, 2),
                                      (64, 0), (1, 0), (2, 2), (7, 6), (130, 130), (16, 16), (24, 8), (8, 8), (136, 64)])
def test_head_dims(B, dim, dims, interleaved, dt):
    rng = np.random.default_rng(dim * 300 + dims)
    for n, heads, normed in ((1, 1, False), (5, 3, True), (67, 2, True), (130, 1, False)):
        norm = (1 + 0.3 * rng.standard_normal(dim)).astype(np.float32) if normed else None
        run(B, draw(rng, (n, heads, dim), dt), rng.integers(0, 5000, n), dims, dt, interleaved, norm=norm)


LAYOUTS = ["tokens", "features", "heads", "gaps", "wide", "odd"]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("out", LAYOUTS)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_strides(B, layout, out, dt):
    rng = np.random.default_rng(1)
    for n, heads, dim, dims, interleaved in ((33, 5, 64, 64, False), (70, 3, 128, 64, True), (3, 9, 80, 80, False)):
        norm = (1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)
        x = draw(rng, (n, heads, dim), dt)
        run(B, x, rng.integers(0, 900, n), dims, dt, interleaved, norm=norm, layout=layout, out=out)
        if layout == out:
            run(B, x, rng.integers(0, 900, n), dims, dt, interleaved, layout=layout, inplace=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_numbers_of_tokens_and_heads(B, dt):
    rng = np.random.default_rng(2)
    for n, heads in ((1, 64), (2, 1), (15, 7), (16, 16), (17, 40), (63, 2), (64, 3), (65, 1), (1000, 12), (4097, 2), (1, 1000)):
        for layout in ("tokens", "features"):
            run(B, draw(rng, (n, heads, 64), dt), rng.integers(0, 70000, n), 64, dt, layout=layout, out=layout)


@pytest.mark.parametrize("pos", [0, 1, -1, -12345, 1 << 20, (1 << 30) - 1, 2 ** 31 - 1, -2 ** 31])
def test_far_positions(B, pos):
    rng = np.random.default_rng(3)
    for layout in ("tokens", "features"):
        run(B, draw(rng, (3, 2, 64), "f32"), [pos, 0, pos], 64, "f32", layout=layout)


def test_turned_back(B):
    """A rotation by -p undoes one by p."""
    import torch
    rng = np.random.default_rng(4)
    x, pos = draw(rng, (9, 3, 64), "f32"), rng.integers(0, 1 << 20, 9)
    y = run(B, x, pos, 64, "f32")
    z = run(B, y.cpu().numpy(), -pos, 64, "f32")
    assert torch.allclose(z.cpu(), torch.from_numpy(x), atol=4e-6)   # two rotations of values up to 4, 16 2^-24 of their sum each


@pytest.mark.parametrize("scaling", [None, (4.0, 0.0, 0.0, 0.0, 0), (8.0, 8192.0, 1.0, 4.0, 1), (4.0, 32768.0, 1.0, 32.0, 2)])
def test_scaled(B, scaling):
    rng = np.random.default_rng(5)
    freq = B.bsp_rope_freqs(64, 500000.0, None if scaling is None else B.RopeScaling(*scaling))
    assert np.allclose(freq, S.freqs(64, 500000.0, *(scaling or ())), rtol=1e-12, atol=0)
    run(B, draw(rng, (20, 2, 64), "f32"), rng.integers(0, 100000, 20), 64, "f32", freq=freq, factor=1.25)


def test_norm_of_nothing_and_of_large_values(B):
    x = np.zeros((3, 2, 64), np.float32)
    x[1] = 1e15
    norm = np.ones(64, np.float32)
    for layout in ("tokens", "features"):
        y = run(B, x, [5, 6, 7], 32, "f32", norm=norm, eps=1e-6, layout=layout, out=layout)
        assert (y[0].cpu().numpy() == 0).all()


class Cache:
    def __init__(self, B, rng, seqs, width, pages, page, kv, dim, dt, order):
        import torch
        inner = (kv, page) if order == "heads" else (page, kv)
        self.data = torch.full((2, pages, *inner, dim), float("nan"), dtype=tdt(dt), device="cuda")
        self.shape = B.CacheShape.of(self.data[0], B.HEAD_MAJOR if order == "heads" else B.SLOT_MAJOR)
        self.table = np.full((seqs, width), -1, np.int64)
        ids = rng.permutation(pages)[:seqs * width]
        self.table.flat[:len(ids)] = ids
        self.page, self.order = page, order

    def slots(self):
        """[2, page, slot, kv, dim]"""
        return self.data if self.order == "slots" else self.data.transpose(2, 3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["heads", "slots"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,heads,kv,dim,dims,page,normed", [(1, 8, 2, 64, 64, 16, False), (33, 6, 3, 128, 128, 16, True), (70, 3, 1, 80, 40, 7, True),
                                                             (200, 4, 4, 96, 96, 64, False), (19, 5, 1, 256, 64, 1, True), (9, 2, 2, 8, 8, 3, True)])
def test_into_the_cache(B, n, heads, kv, dim, dims, page, normed, layout, order, dt):
    import torch
    rng = np.random.default_rng(n)
    seqs, width = 5, M.ceil(n, page) + 1
    c = Cache(B, rng, seqs, width, seqs * width + 3, page, kv, dim, dt, order)
    rows = rng.integers(0, seqs, n)
    pos = np.array([rng.permutation(width * page)[i] for i in range(n)])
    seen = set()
    for i in range(n):   # a place of its own for each; some that have none
        pos[i] = -1 if (rows[i], pos[i]) in seen else pos[i]
        seen.add((rows[i], pos[i]))
    if n > 8:
        pos[3], pos[4], rows[5], rows[6] = width * page, -7, seqs, -1
        c.table[rows[7], pos[7] // page] = -1
        c.table[rows[8], pos[8] // page] = 10 ** 6
    before = c.data.clone()
    q, k, v = (draw(rng, (n, h, dim), dt) for h in (heads, kv, kv))
    qn, kn = ((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32) if normed else None for _ in range(2))
    freq = S.freqs(dims, 10000.0)
    interleaved = n % 2 == 0
    rope = B.Rope(B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, dims)
    qd, kd, vd = (place(a, dt, layout) for a in (q, k, v))
    out = place(np.full_like(q, np.nan), dt, layout)
    dev = [None if a is None else torch.from_numpy(a).cuda() for a in (qn, kn)]
    B.bsp_cache_append_rotary(c.shape, rope, torch.tensor(freq, dtype=torch.float64, device="cuda"), qd, kd, vd, out, c.data[0],
                              c.data[1], ints(c.table), ints(pos), ints(rows), *dev, 1e-5)
    torch.cuda.synchronize()
    close(out, *S.rotate(q, pos, freq, interleaved, 1.0, qn, 1e-5), dt)
    want, bound = S.rotate(k, pos, freq, interleaved, 1.0, kn, 1e-5)
    slots, written = c.slots(), torch.zeros(c.slots().shape[1:3], dtype=torch.bool)
    for i in range(n):
        if not (0 <= rows[i] < seqs and 0 <= pos[i] < width * page):
            continue
        p = c.table[rows[i], pos[i] // page]
        if not 0 <= p < c.data.shape[1]:
            continue
        s = int(pos[i] % page)
        written[p, s] = True
        close(slots[0, p, s], want[i], bound[i], dt)
        assert (slots[1, p, s].float().cpu().numpy() == v[i]).all()
    old = before if order == "slots" else before.transpose(2, 3)
    assert bool(slots[:, ~written].isnan().all()) and bool(old[:, ~written].isnan().all())   # nothing else is written
    # in place, and the default rows
    m = min(n, seqs)
    r = np.arange(m) % width * page % (width * page)
    B.bsp_cache_append_rotary(c.shape, rope, torch.tensor(freq, dtype=torch.float64, device="cuda"), qd[:m], kd[:m], vd[:m], qd[:m],
                              c.data[0], c.data[1], ints(c.table), ints(r), None, *dev, 1e-5)
    torch.cuda.synchronize()
    close(qd[:m], *S.rotate(q[:m], r, freq, interleaved, 1.0, qn, 1e-5), dt)


def test_an_offset_past_32_bits(B):
    """A page 2^31 elements into the cache."""
    import torch
    rng = np.random.default_rng(6)
    page, kv, dim = 64, 8, 128
    pages = (1 << 31) // (page * kv * dim) + 2
    keys, values = (torch.empty(pages, kv, page, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    shape = B.CacheShape.of(keys)
    x = draw(rng, (1, kv, dim), "bf16")
    d = place(x, "bf16", "tokens")
    out, freq = torch.empty_like(d), S.freqs(dim, 10000.0)
    B.bsp_cache_append_rotary(shape, B.Rope(0, dim), torch.tensor(freq, dtype=torch.float64, device="cuda"), d, d, d, out, keys, values,
                              ints([[3, pages - 1]]), ints([page + 5]))
    torch.cuda.synchronize()
    assert (values[pages - 1, :, 5].cpu() == d[0].cpu()).all() and (keys[pages - 1, :, 5].cpu() == out[0].cpu()).all()
    close(out, *S.rotate(x, [page + 5], freq, False, 1.0, None, 0), "bf16")


def test_streams_and_graphs(B):
    import torch
    rng = np.random.default_rng(7)
    stream = torch.cuda.Stream()
    run(B, draw(rng, (40, 4, 64), "bf16"), np.arange(40), 64, "bf16", stream=stream)
    x = draw(rng, (40, 4, 64), "bf16")
    xd, pos, y = place(x, "bf16", "features"), ints(np.arange(40)), place(x, "bf16", "features")
    freq = S.freqs(64, 10000.0)
    fd, graph = torch.tensor(freq, dtype=torch.float64, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.bsp_rotary(B.BF16, B.Rope(0, 64), fd, xd, pos, y)
    for turn in range(3):
        pos += 100 * turn
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        close(y, *S.rotate(x, pos.cpu().numpy(), freq, False, 1.0, None, 0), "bf16")
