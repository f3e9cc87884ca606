"""What rotary positions, attention over a shared prefix and sampling refuse, their size queries, and the
frequencies.  CPU only: no call here launches a kernel."""

import ctypes
import math

import pytest

from tests import sampling_model as S
from tests.test_decode_abi import EINVAL, EUNSUPPORTED, P4, P16, B, L, cache   # noqa: F401 (B and L are fixtures)

P2 = ctypes.c_void_p(4098)


@pytest.mark.parametrize("dims", [0, 2, 40, 64, 128])
@pytest.mark.parametrize("scaling", [None, (4.0, 0.0, 0.0, 0.0, 0), (8.0, 8192.0, 1.0, 4.0, 1), (4.0, 32768.0, 1.0, 32.0, 2),
                                     (16.0, 4096.0, 1.0, 32.0, 2), (2.0, 100.0, 0.5, 0.6, 1), (2.0, 10.0, 1.0, 1e9, 2)])
def test_freqs(B, dims, scaling):
    got = B.bsp_rope_freqs(dims, 10000.0, None if scaling is None else B.RopeScaling(*scaling))
    want = S.freqs(dims, 10000.0, *(scaling or ()))
    assert len(got) == dims // 2 and all(abs(a - b) <= 1e-13 * b for a, b in zip(got, want))


def test_freqs_refusals(B, L):
    out = (ctypes.c_double * 64)()
    a = ctypes.addressof(out)

    def call(dims=64, base=1e4, out=a, **kw):
        c = dict(factor=2.0, original=100.0, low=1.0, high=4.0, ramp=1)
        c.update(kw)
        return L.bsp_rope_freqs(dims, base, B.RopeScaling(*c.values()), out)
    assert call() == 0 and call(dims=0, out=None) == 0 and call(ramp=2) == 0 and call(ramp=0, original=0.0, low=0.0, high=0.0) == 0
    assert call(dims=-2) == EINVAL and call(dims=3) == EINVAL and call(out=None) == EINVAL
    for base in (0.0, -1.0, math.inf, math.nan):
        assert call(base=base) == EINVAL and L.bsp_rope_freqs(64, base, None, a) == EINVAL
    for factor in (0.0, -1.0, math.nan, math.inf):
        assert call(factor=factor) == EINVAL
    assert call(ramp=3) == EINVAL and call(ramp=-1) == EINVAL
    for ramp in (1, 2):
        for bad in (dict(original=0.0), dict(original=math.nan), dict(original=math.inf), dict(low=4.0), dict(low=5.0), dict(low=math.nan),
                    dict(high=math.inf), dict(high=math.nan), dict(low=-math.inf)):
            assert call(ramp=ramp, **bad) == EINVAL
    assert call(ramp=2, low=0.0) == EINVAL and call(ramp=2, low=-1.0) == EINVAL and call(ramp=2, base=1.0) == EINVAL
    with pytest.raises(B.BspError):
        B.bsp_rope_freqs(3, 1e4)


def test_rotary_refusals(B, L):
    s = B._Strides(128, 64, 1)

    def call(dt=1, rope=(0, 64, 1.0), freqs=P16, n=2, heads=4, dim=64, x=P16, xs=s, pos=P16, norm=None, eps=1e-6, y=P16, ys=s):
        return L.bsp_rotary(dt, None if rope is None else B.Rope(*rope), freqs, n, heads, dim, x, xs, pos, norm, eps, y, ys, None)
    assert call(n=0) == 0 and call(n=0, rope=(1, 0, 1.0), freqs=None) == 0
    assert call(dt=2) == EINVAL and call(rope=None) == EINVAL and call(n=-1) == EINVAL and call(heads=0) == EINVAL and call(dim=0) == EINVAL
    assert call(rope=(2, 64, 1.0)) == EINVAL and call(rope=(0, 63, 1.0)) == EINVAL and call(rope=(0, -2, 1.0)) == EINVAL
    assert call(rope=(0, 66, 1.0)) == EINVAL and call(freqs=None) == EINVAL and call(freqs=P4) == EINVAL
    assert call(x=None) == EINVAL and call(y=None) == EINVAL and call(pos=None) == EINVAL and call(xs=None) == EINVAL and call(ys=None) == EINVAL
    assert call(dt=0, x=P2) == EINVAL and call(dt=0, y=P2) == EINVAL and call(x=ctypes.c_void_p(4097)) == EINVAL and call(pos=P2) == EINVAL
    assert call(norm=P2) == EINVAL and call(norm=P16, eps=-1.0) == EINVAL and call(norm=P16, eps=math.nan) == EINVAL
    assert call(dim=257) == EUNSUPPORTED and call(heads=65536) == EUNSUPPORTED and call(n=1 << 24) == EUNSUPPORTED


def test_append_rotary_refusals(B, L):
    c, s = cache(B), B._Strides(128, 64, 1)

    def call(cache=c, rope=(0, 64, 1.0), freqs=P16, n=2, heads=4, q=P16, qs=s, k=P16, ks=s, v=P16, vs=s, out=P16, outs=s, qn=None, kn=None,
             eps=1e-6, keys=P16, values=P16, table=P16, seqs=2, width=4, rows=None, pos=P16):
        return L.bsp_cache_append_rotary(cache, B.Rope(*rope), freqs, n, heads, q, qs, k, ks, v, vs, out, outs, qn, kn, eps, keys, values, table,
                                         seqs, width, rows, pos, None)
    assert call(n=0) == 0
    for bad in (dict(cache=None), dict(rope=(0, 66, 1.0)), dict(rope=(3, 2, 1.0)), dict(freqs=None), dict(n=-1), dict(heads=0), dict(q=None),
                dict(qs=None), dict(k=None), dict(ks=None), dict(v=None), dict(vs=None), dict(out=None), dict(outs=None), dict(qn=P2), dict(kn=P2),
                dict(qn=P16, eps=-1.0), dict(kn=P16, eps=math.nan), dict(keys=None), dict(keys=P4), dict(values=P4), dict(table=None), dict(seqs=-1),
                dict(width=-1), dict(rows=P2), dict(pos=None), dict(pos=P2), dict(q=ctypes.c_void_p(4097)), dict(v=ctypes.c_void_p(4097))):
        assert call(**bad) == EINVAL, bad
    assert call(heads=65532) == EUNSUPPORTED and call(n=1 << 24) == EUNSUPPORTED and call(width=1 << 28) == EUNSUPPORTED
    assert call(cache=cache(B, head_dim=60)) == EUNSUPPORTED and call(cache=cache(B, dtype=2)) == EINVAL


def test_prefix_refusals(B, L):
    c, s, out = cache(B), B._Strides(128, 64, 1), ctypes.c_int64()
    a = ctypes.addressof(out)

    def call(cache=c, batch=2, heads=4, q=P16, qs=s, keys=P16, values=P16, table=P16, seqs=2, width=4, rows=None, lens=P16, groups=1, starts=P16,
             shared=P16, prefix=None, window=0, y=P16, ys=s, lse=None, ws=P16):
        return L.bsp_attention_prefix(cache, batch, heads, q, qs, keys, values, table, seqs, width, rows, lens, groups, starts, shared, prefix, 1.0,
                                      window, y, ys, lse, ws, None)
    assert call(batch=0, groups=0) == 0
    for bad in (dict(cache=None), dict(batch=-1), dict(heads=0), dict(heads=3), dict(q=None), dict(qs=None), dict(ys=None), dict(y=None),
                dict(keys=None), dict(keys=P4), dict(values=P4), dict(table=None), dict(seqs=-1), dict(width=-1), dict(lens=None), dict(groups=-1),
                dict(starts=None), dict(shared=None), dict(window=-1), dict(lse=P2), dict(starts=P2), dict(shared=P2), dict(prefix=P2), dict(rows=P2),
                dict(lens=P2), dict(table=P2), dict(q=ctypes.c_void_p(4097)), dict(y=ctypes.c_void_p(4097))):
        assert call(**bad) == EINVAL, bad
    assert call(batch=1025) == EUNSUPPORTED and call(groups=3) == EUNSUPPORTED and call(width=1 << 28) == EUNSUPPORTED
    assert call(cache=cache(B, head_dim=264)) == EUNSUPPORTED
    q = L.bsp_attention_prefix_workspace
    assert q(c, 2, 3, 1, 4, a) == EINVAL and q(c, -1, 4, 0, 4, a) == EINVAL and q(c, 2, 4, 1, 4, None) == EINVAL and q(c, 2, 4, -1, 4, a) == EINVAL
    assert q(c, 1025, 4, 1, 4, a) == EUNSUPPORTED and q(c, 2, 4, 3, 4, a) == EUNSUPPORTED and q(c, 2, 4, 1, 1 << 28, a) == EUNSUPPORTED
    assert q(c, 0, 2, 0, 0, a) == 0 and out.value >= 0
    for batch, heads, groups, width in ((1024, 64, 1024, 1 << 20), (64, 64, 1, 2048), (1, 2, 0, 1)):
        assert q(c, batch, heads, groups, width, a) == 0
        if out.value > 0:
            assert call(batch=batch, heads=heads, groups=groups, width=width, seqs=batch, ws=None) == EINVAL
            assert call(batch=batch, heads=heads, groups=groups, width=width, seqs=batch, ws=P4) == EINVAL


def test_sample_refusals(L):
    out = ctypes.c_int64()
    a = ctypes.addressof(out)

    def call(dt=0, batch=2, vocab=100, logits=P16, u=P16, t=None, k=None, p=None, m=None, tokens=P16, logp=None, ws=P16):
        return L.bsp_sample(dt, batch, vocab, logits, vocab, 1, u, t, k, p, m, tokens, logp, ws, None)
    assert call(batch=0) == 0 and call(batch=0, logits=None, u=None, tokens=None, ws=None) == 0
    for bad in (dict(dt=2), dict(batch=-1), dict(vocab=0), dict(logits=None), dict(u=None), dict(tokens=None), dict(logits=P2), dict(u=P2), dict(t=P2),
                dict(k=P2), dict(p=P2), dict(m=P2), dict(tokens=P2), dict(logp=P2), dict(dt=1, logits=ctypes.c_void_p(4097))):
        assert call(**bad) == EINVAL, bad
    assert call(vocab=(1 << 20) + 1) == EUNSUPPORTED and call(batch=1 << 24) == EUNSUPPORTED and call(batch=1 << 12, vocab=1 << 20) == EUNSUPPORTED
    q = L.bsp_sample_workspace
    assert q(2, 0, a) == EINVAL and q(-1, 5, a) == EINVAL and q(2, 5, None) == EINVAL
    assert q(2, (1 << 20) + 1, a) == EUNSUPPORTED and q(1 << 12, 1 << 20, a) == EUNSUPPORTED and q(0, 5, a) == 0
    for batch, vocab in ((1, 1), (3, 1 << 20), (64, 131072), (2047, 1 << 20)):
        assert q(batch, vocab, a) == 0
        if out.value > 0:
            assert call(batch=batch, vocab=vocab, ws=None) == EINVAL and call(batch=batch, vocab=vocab, ws=P4) == EINVAL


def test_the_binding_refuses_host_arrays_and_wrong_types(B):
    import torch
    x, pos = torch.zeros(2, 3, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    rope = B.Rope(B.ROPE_HALF, 64)
    freqs = torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="device"):
        B.bsp_rotary(B.BF16, rope, freqs, x, pos, x)
    with pytest.raises(ValueError, match="type"):
        B.bsp_rotary(B.F32, rope, freqs, x, pos, x)
    with pytest.raises(ValueError, match="y must be"):
        B.bsp_rotary(B.BF16, rope, freqs, x, pos, x[:1])
    with pytest.raises(ValueError, match="tokens, heads"):
        B.bsp_rotary(B.BF16, rope, freqs, x[0], pos, x[0])
    with pytest.raises(ValueError, match="type"):
        B.bsp_sample(B.F32, torch.zeros(2, 5, dtype=torch.float16), pos, pos)
    with pytest.raises(ValueError, match="batch, vocab"):
        B.bsp_sample(B.F32, torch.zeros(5), pos, pos)
    with pytest.raises(ValueError, match="device"):
        B.bsp_sample(B.F32, torch.zeros(2, 5), pos, pos)
