"""What the decode operators refuse, and their size queries.  CPU only: no call here launches a kernel."""

import ctypes
import os

import pytest

EINVAL, EUNSUPPORTED = -1, -2
P16, P4 = ctypes.c_void_p(4096), ctypes.c_void_p(4100)   # never followed: the calls fail before


@pytest.fixture(scope="module")
def B():
    import paper_2111_11581_amd as B
    if not os.path.exists(B.lib_path()):
        from paper_2111_11581_amd import build
        build.build()
    B.lib()
    return B


@pytest.fixture
def L(B):
    return B.lib()


def cache(B, **kw):
    c = dict(dtype=1, order=0, pages=10, page_size=16, kv_heads=2, head_dim=64, page_stride=0)
    c.update(kw)
    return B.CacheShape(*[c[k] for k in ("dtype", "order", "pages", "page_size", "kv_heads", "head_dim", "page_stride")])


@pytest.mark.parametrize("rows,cols,group,want", [
    (1, 1, 32, (16, 16)), (4099, 1003, 32, (4099 * 512, 32 * 4112)), (16, 128, 128, (16 * 64, 16)),
    (17, 129, 64, (17 * 80, 3 * 32)), (70000, 70000, 128, (70000 * 35008, 547 * 70000))])
def test_q4_sizes(B, rows, cols, group, want):
    assert B.bsp_q4_sizes(rows, cols, group) == want


@pytest.mark.parametrize("rows,cols,group", [(0, 8, 32), (8, 0, 32), (-1, 8, 32), (8, 8, 0), (8, 8, 16), (8, 8, 96), (8, 8, 256)])
def test_q4_refusals(B, L, rows, cols, group):
    out = (ctypes.c_int64 * 2)()
    a = ctypes.addressof(out)
    assert L.bsp_q4_sizes(rows, cols, group, a, a + 8) == EINVAL
    assert L.bsp_q4_quantize(rows, cols, group, 1, P16, None, P16, P16, None) == EINVAL
    assert L.bsp_q4_dequantize(rows, cols, group, 1, P16, P16, P16, None) == EINVAL
    assert L.bsp_q4_linear(rows, cols, group, 1, 1, 1, P16, P16, P16, None, 0, P16, None) == EINVAL
    with pytest.raises(B.BspError):
        B.bsp_q4_sizes(rows, cols, group)


def test_q4_linear_refusals(L):
    def call(batch=4, in_dt=1, out_dt=1, x=P16, codes=P16, scales=P16, bias=None, y=P16, rows=64, cols=64):
        return L.bsp_q4_linear(rows, cols, 64, batch, in_dt, out_dt, x, codes, scales, bias, 0, y, None)
    assert call(batch=0) == 0
    assert call(batch=-1) == EINVAL
    assert call(in_dt=2) == EINVAL and call(out_dt=-1) == EINVAL
    assert call(x=None) == EINVAL and call(codes=None) == EINVAL and call(scales=None) == EINVAL and call(y=None) == EINVAL
    assert call(codes=P4) == EINVAL and call(scales=P4) == EINVAL
    assert call(in_dt=0, x=ctypes.c_void_p(4098)) == EINVAL and call(bias=ctypes.c_void_p(4098)) == EINVAL
    assert call(batch=1 << 26) == EUNSUPPORTED


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=2), EINVAL), (dict(order=2), EINVAL), (dict(pages=0), EINVAL), (dict(page_size=0), EINVAL),
    (dict(kv_heads=0), EINVAL), (dict(head_dim=0), EINVAL), (dict(head_dim=60), EUNSUPPORTED),
    (dict(head_dim=264), EUNSUPPORTED), (dict(page_stride=16 * 2 * 64 - 8), EINVAL), (dict(page_stride=16 * 2 * 64 + 4), EINVAL),
    (dict(page_stride=-8), EINVAL), (dict(page_size=1 << 23), EUNSUPPORTED)])
def test_cache_refusals(B, L, bad, status):
    c, s, out = cache(B, **bad), B._Strides(128, 64, 1), ctypes.c_int64()
    a = ctypes.addressof(out)
    assert L.bsp_attention_workspace(c, 1, 2, 4, a) == status
    assert L.bsp_cache_scratch(c, 1, 4, 1, a) == status
    assert L.bsp_cache_append(c, 1, P16, s, P16, s, P16, P16, P16, 1, 4, None, P16, None) == status
    assert L.bsp_attention(c, 1, 2, P16, s, P16, P16, P16, 1, 4, None, P16, 1.0, 0, P16, s, None, P16, None) == status
    assert L.bsp_cache_extend(c, 1, 0, P16, 1, 4, P16, P16, P16, 1, P16, P16, P16, P16, None) == status
    assert L.bsp_cache_compact(c, 1, 0, P16, 1, 4, P16, P16, P16, P16, None) == status
    assert L.bsp_cache_copy(c, 1, 0, P16, 1, P16, P16, None) == status


def test_attention_refusals(B, L):
    c, s = cache(B), B._Strides(128, 64, 1)

    def call(cache=c, batch=2, heads=4, q=P16, qs=s, keys=P16, values=P16, table=P16, seqs=2, width=4, lens=P16, window=0,
             y=P16, ys=s, ws=P16):
        return L.bsp_attention(cache, batch, heads, q, qs, keys, values, table, seqs, width, None, lens, 1.0, window, y, ys,
                               None, ws, None)
    assert call(batch=0) == 0
    assert call(cache=None) == EINVAL and call(qs=None) == EINVAL and call(ys=None) == EINVAL
    assert call(batch=-1) == EINVAL and call(heads=0) == EINVAL and call(heads=3) == EINVAL and call(window=-1) == EINVAL
    assert call(q=None) == EINVAL and call(y=None) == EINVAL and call(keys=None) == EINVAL and call(values=None) == EINVAL
    assert call(table=None) == EINVAL and call(lens=None) == EINVAL and call(seqs=-1) == EINVAL and call(width=-1) == EINVAL
    assert call(keys=P4) == EINVAL and call(values=P4) == EINVAL
    assert call(width=1 << 28) == EUNSUPPORTED and call(batch=1 << 22) == EUNSUPPORTED
    out = ctypes.c_int64()
    a = ctypes.addressof(out)
    assert L.bsp_attention_workspace(c, 2, 3, 4, a) == EINVAL and L.bsp_attention_workspace(c, -1, 2, 4, a) == EINVAL
    assert L.bsp_attention_workspace(c, 2, 2, 4, None) == EINVAL
    assert L.bsp_attention_workspace(c, 0, 2, 0, a) == 0


def test_append_refusals(B, L):
    c, s = cache(B), B._Strides(128, 64, 1)

    def call(cache=c, n=2, k=P16, ks=s, v=P16, vs=s, keys=P16, values=P16, table=P16, seqs=2, width=4, pos=P16):
        return L.bsp_cache_append(cache, n, k, ks, v, vs, keys, values, table, seqs, width, None, pos, None)
    assert call(n=0) == 0 and call(seqs=0) == 0
    assert call(n=-1) == EINVAL and call(k=None) == EINVAL and call(v=None) == EINVAL and call(pos=None) == EINVAL
    assert call(ks=None) == EINVAL and call(vs=None) == EINVAL and call(table=None) == EINVAL
    assert call(keys=P4) == EINVAL and call(values=None) == EINVAL
    assert call(width=1 << 28) == EUNSUPPORTED


def test_pages_refusals(B, L):
    c = cache(B)

    def fork(seqs=2, width=4, pages=10, table=P16, lens=P16, refs=P16, n=1, parents=P16, children=P16, scratch=P16):
        return L.bsp_cache_fork(seqs, width, pages, table, lens, refs, n, parents, children, scratch, None)

    def release(seqs=2, width=4, pages=10, table=P16, lens=P16, refs=P16, n=1, rows=P16):
        return L.bsp_cache_release(seqs, width, pages, table, lens, refs, n, rows, None)
    for f in (fork, release):
        assert f(n=0) == 0 and f(seqs=0) == 0
        assert f(n=-1) == EINVAL and f(seqs=-1) == EINVAL and f(width=-1) == EINVAL and f(pages=0) == EINVAL
        assert f(table=None) == EINVAL and f(lens=None) == EINVAL and f(refs=None) == EINVAL
    assert fork(parents=None) == EINVAL and fork(children=None) == EINVAL and fork(scratch=None) == EINVAL
    assert fork(scratch=P4) == EINVAL and release(rows=None) == EINVAL

    def extend(planes=2, stride=1 << 16, data=P16, seqs=2, width=4, table=P16, lens=P16, refs=P16, n=1, rows=P16, counts=P16,
               pos=P16, scratch=P16):
        return L.bsp_cache_extend(c, planes, stride, data, seqs, width, table, lens, refs, n, rows, counts, pos, scratch, None)
    assert extend(n=0) == 0
    assert extend(planes=-1) == EINVAL and extend(stride=-8) == EINVAL and extend(stride=4) == EINVAL
    assert extend(data=None) == EINVAL and extend(data=P4) == EINVAL and extend(refs=None) == EINVAL
    assert extend(rows=None) == EINVAL and extend(counts=None) == EINVAL and extend(pos=None) == EINVAL
    assert extend(scratch=None) == EINVAL and extend(n=-2) == EINVAL and extend(width=1 << 28) == EUNSUPPORTED

    def compact(planes=2, data=P16, table=P16, refs=P16, info=P16, scratch=P16, seqs=2):
        return L.bsp_cache_compact(c, planes, 1 << 16, data, seqs, 4, table, refs, info, scratch, None)
    assert compact(data=None) == EINVAL and compact(table=None) == EINVAL and compact(refs=None) == EINVAL
    assert compact(info=None) == EINVAL and compact(scratch=None) == EINVAL and compact(seqs=-1) == EINVAL
    assert L.bsp_cache_copy(c, 2, 1 << 16, P16, 0, None, None, None) == 0
    assert L.bsp_cache_copy(c, 2, 1 << 16, P16, -1, P16, P16, None) == EINVAL
    assert L.bsp_cache_copy(c, 2, 1 << 16, P16, 1, None, P16, None) == EINVAL


def test_the_binding_refuses_host_arrays_and_wrong_shapes(B):
    import torch
    with pytest.raises(ValueError):
        B.bsp_q4_linear(16, 32, 32, 1, 1, 1, torch.zeros(32, 1, dtype=torch.bfloat16), torch.zeros(256, dtype=torch.uint8),
                        torch.zeros(16, dtype=torch.bfloat16), None, False, torch.zeros(16, 1, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.bsp_q4_dequantize(16, 32, 32, 1, torch.zeros(10, dtype=torch.uint8), torch.zeros(16, dtype=torch.bfloat16),
                            torch.zeros(16, 32, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        B.CacheShape.of(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16))       # on the host
    with pytest.raises(ValueError):
        B.CacheShape.of(torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16).transpose(1, 2))
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.bsp_cache_release(t, t[0], t[0], t[0])


def test_q4_of_more_than_one_launch_is_refused(L):
    big = (1 << 26) + 1
    assert L.bsp_q4_quantize(big, 2048, 64, 1, P16, None, P16, P16, None) == EUNSUPPORTED
    assert L.bsp_q4_dequantize(2048, big, 64, 1, P16, P16, P16, None) == EUNSUPPORTED
    assert L.bsp_q4_linear(big, 64, 64, 1, 1, 1, P16, P16, P16, None, 0, P16, None) == EUNSUPPORTED
    assert L.bsp_q4_linear(64, big, 64, 1, 1, 1, P16, P16, P16, None, 0, P16, None) == EUNSUPPORTED
    assert L.bsp_q4_linear(1, 1, 64, (1 << 19) + 1, 1, 1, P16, P16, P16, None, 0, P16, None) == EUNSUPPORTED
    assert L.bsp_q4_quantize(2**31 - 1, 1, 64, 1, P16, None, P16, P16, None) == EINVAL
