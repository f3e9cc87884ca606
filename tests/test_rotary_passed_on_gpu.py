"""Dimensions that a rotation passes on keep their bits, whatever they hold and however the arrays lie, and nothing
of them reaches those that are rotated."""

import numpy as np
import pytest

from tests.test_rotary_gpu import B, ints, place, tdt   # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


def bits(t):
    import torch
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def odd_values(rng, n, dt):
    """Infinities, NaN of several kinds, zeros of both signs, denormals and ordinary numbers, as bits."""
    inf, quiet, least = (0x7f80, 0x40, 1) if dt == "bf16" else (0x7f800000, 0x400000, 0x10000)
    kinds = np.array([inf, inf | quiet, inf | quiet | 5 * least, inf | least, 0, least, inf // 2], np.int64)
    out = kinds[rng.integers(0, len(kinds), n)]
    top = 1 << (15 if dt == "bf16" else 31)
    return np.where(rng.random(n) < 0.5, out - top, out).astype(np.int16 if dt == "bf16" else np.int32)


def arrays(rng, n, heads, dim, dims, dt):
    """[n, heads, dim] twice, alike in the rotated dimensions and ordinary and odd in the others."""
    import torch
    a = torch.from_numpy(rng.standard_normal((n, heads, dim)).astype(np.float32)).to(tdt(dt))
    b = a.clone()
    b[:, :, dims:] = torch.from_numpy(odd_values(rng, n * heads * (dim - dims), dt)).view(tdt(dt)).view(n, heads, dim - dims)
    return a, b


def put(t, dt, layout):
    """As place(), by bits."""
    out = place(np.zeros(t.shape, np.float32), dt, layout)
    out.copy_(t)
    assert np.array_equal(bits(out).cpu().numpy(), bits(t).numpy())
    return out


@pytest.mark.parametrize("layout", ["tokens", "wide", "gaps", "features"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dt,dim,dims", [("bf16", 24, 8), ("bf16", 80, 40), ("bf16", 64, 24), ("bf16", 256, 248), ("bf16", 96, 32), ("bf16", 72, 6),
                                         ("f32", 12, 4), ("f32", 80, 20), ("f32", 256, 252), ("f32", 64, 32), ("f32", 40, 10)])
def test_passed_on(B, dt, dim, dims, interleaved, layout):
    import torch
    rng = np.random.default_rng(dim + dims)
    rope = B.Rope(B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, dims, 1.5)
    freqs = torch.tensor(B.bsp_rope_freqs(dims, 1e4), dtype=torch.float64, device="cuda")
    for n, heads in ((1, 1), (3, 5), (70, 2), (210, 3)):
        pos, out = ints(rng.integers(0, 5000, n)), []
        for x in arrays(rng, n, heads, dim, dims, dt):
            for inplace in (False, True):
                xd = put(x, dt, layout)
                yd = xd if inplace else put(torch.zeros_like(x), dt, layout)
                B.bsp_rotary(B.BF16 if dt == "bf16" else B.F32, rope, freqs, xd, pos, yd)
                torch.cuda.synchronize()
                got = bits(yd).cpu()
                assert torch.equal(got[:, :, dims:], bits(x)[:, :, dims:]), (n, heads, inplace)
                out.append(got[:, :, :dims])
        assert all(torch.equal(out[0], o) for o in out[1:])


@pytest.mark.parametrize("dt,dim,dims", [("bf16", 24, 8), ("bf16", 128, 40), ("f32", 16, 4), ("f32", 128, 20)])
def test_passed_on_into_the_cache(B, dt, dim, dims):
    import torch
    rng = np.random.default_rng(dim)
    freqs = torch.tensor(B.bsp_rope_freqs(dims, 1e4), dtype=torch.float64, device="cuda")
    rope = B.Rope(B.ROPE_INTERLEAVED, dims)
    for n in (1, 9, 70):
        pages = -(-n // 4)
        (q, q2), (k, k2), (_, v) = (arrays(rng, n, h, dim, d, dt) for h, d in ((4, dims), (2, dims), (2, 0)))
        table, pos, out = ints([list(range(pages))]), ints(range(n)), []
        rows = ints([0] * n)
        for a, b in ((q, k), (q2, k2)):
            data = torch.zeros(2, pages, 4, 2, dim, dtype=tdt(dt), device="cuda")
            y = torch.zeros(n, 4, dim, dtype=tdt(dt), device="cuda")
            cache = B.CacheShape.of(data[0], B.SLOT_MAJOR)
            B.bsp_cache_append_rotary(cache, rope, freqs, a.cuda(), b.cuda(), v.cuda(), y, *data, table, pos, rows)
            torch.cuda.synchronize()
            keys, values = (bits(p).cpu().view(-1, 2, dim)[:n] for p in data)
            assert torch.equal(bits(y).cpu()[:, :, dims:], bits(a)[:, :, dims:]) and torch.equal(keys[:, :, dims:], bits(b)[:, :, dims:])
            assert torch.equal(values, bits(v))
            out.append((bits(y).cpu()[:, :, :dims], keys[:, :, :dims]))
        assert all(torch.equal(x, y) for x, y in zip(*out))
