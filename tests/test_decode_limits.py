"""Limits of the decode operators: sizes, alignment, layouts and types at which a call has to be refused
or to ask for more.  CPU only: no call here launches a kernel."""

import ctypes

import pytest

from tests.test_decode_abi import EINVAL, EUNSUPPORTED, P16, B, L, cache   # noqa: F401 (B and L are fixtures)


def workspace(L, c, batch, heads, width):
    out = ctypes.c_int64(-1)
    assert L.bsp_attention_workspace(c, batch, heads, width, ctypes.addressof(out)) == 0
    return out.value


@pytest.mark.parametrize("batch,page,width", [(1024, 1 << 20, 64), (64, 512, 1 << 21), (64, 1 << 16, 1 << 14), (1000, 16, 1 << 26)])
def test_a_window_over_very_long_tables_has_its_workspace(B, L, batch, page, width):
    """The blocks of all sequences together pass 32 bits, those in a window do not."""
    c = cache(B, page_size=page, kv_heads=1, head_dim=64)
    assert workspace(L, c, batch, 1, width) >= workspace(L, c, batch, 1, 4096 * 4 // page + 1) > 0
    s = B._Strides(64, 64, 1)
    for window in (0, 4096, 1 << 20):
        assert L.bsp_attention(c, batch, 1, P16, s, P16, P16, P16, batch, width, None, P16, 1.0, window, P16, s, None, None,
                               None) == EINVAL


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("batch,kv,heads", [(1, 1, 1), (7, 12, 12), (32, 8, 32), (64, 1, 40), (1024, 2, 2), (1025, 2, 2)])
def test_the_workspace_grows_with_the_table(B, L, batch, kv, heads, dtype):
    """So that a call whose window is shorter than its table never needs more than the query said."""
    c = cache(B, dtype=dtype, kv_heads=kv, page_size=64)
    sizes = [workspace(L, c, batch, heads, 1 << k) for k in range(25)]
    assert sizes == sorted(sizes)


def test_types_of_the_same_size_are_told_apart(B):
    import torch
    plane = torch.zeros(4, 2, 16, 64)
    for dtype in (torch.float16, torch.int16, torch.int32, torch.float64, torch.uint8):
        with pytest.raises(ValueError, match="fp32 or bf16"):
            B.CacheShape.of(plane.to(dtype))
    for code, right, wrong in ((B.BF16, torch.bfloat16, (torch.float16, torch.int16, torch.uint16, torch.float32)),
                               (B.F32, torch.float32, (torch.int32, torch.bfloat16, torch.uint32))):
        key = bytes(B.CacheShape(code, B.HEAD_MAJOR, 4, 16, 2, 64, 0))
        page = (tuple(plane.shape), plane.stride())
        B._plane_layout(key, "keys", *page, right)
        B._planes_layout(key, (3, *plane.shape), (plane.numel(), *plane.stride()), right)
        q = ((5, 2, 64), (128, 64, 1))
        B._layouts(key, ("q", "y"), 5, 2, *q, right, *q, right, *page, right, *page, right)
        for dtype in wrong:
            with pytest.raises(ValueError, match="pages"):
                B._plane_layout(key, "keys", *page, dtype)
            with pytest.raises(ValueError, match="pages"):
                B._planes_layout(key, (3, *plane.shape), (plane.numel(), *plane.stride()), dtype)
            for i in range(4):
                types = [dtype if j == i else right for j in range(4)]
                with pytest.raises(ValueError):
                    B._layouts(key, ("q", "y"), 5, 2, *q, types[0], *q, types[1], *page, types[2], *page, types[3])


@pytest.mark.parametrize("dtype,off", [(0, 1), (0, 2), (0, 3), (1, 1)])
def test_arrays_are_aligned_to_their_elements(B, L, dtype, off):
    c, s, odd = cache(B, dtype=dtype), B._Strides(128, 64, 1), ctypes.c_void_p(4096 + off)
    for k, v in ((odd, P16), (P16, odd)):
        assert L.bsp_cache_append(c, 1, k, s, v, s, P16, P16, P16, 1, 4, None, P16, None) == EINVAL
    for q, y, lse in ((odd, P16, None), (P16, odd, None), (P16, P16, ctypes.c_void_p(4098))):
        assert L.bsp_attention(c, 1, 2, q, s, P16, P16, P16, 1, 4, None, P16, 1.0, 0, y, s, lse, P16, None) == EINVAL


@pytest.mark.parametrize("planes,stride,page_stride,ok", [
    (1, 0, 0, True), (0, 0, 0, True), (2, 10 * 2048, 0, True), (2, 10 * 2048 - 8, 0, False), (2, 0, 0, False), (2, 2048, 0, False),
    (3, 9 * 2560 + 2048, 2560, True), (3, 9 * 2560 + 2040, 2560, False),
    (4, 2048, 4 * 2048, True), (4, 2048, 4 * 2048 - 8, False), (4, 2040, 4 * 2048, False), (4, 2056, 4 * 2056, True)])
def test_planes_do_not_overlap(B, L, planes, stride, page_stride, ok):
    """Ten pages of 2048 elements: plane after plane, or pages of all planes beside each other."""
    c = cache(B, page_stride=page_stride)
    want = 0 if ok else EINVAL
    assert L.bsp_cache_copy(c, planes, stride, P16, 0, None, None, None) == want
    assert L.bsp_cache_extend(c, planes, stride, P16, 2, 4, P16, P16, P16, 0, None, None, None, None, None) == want
    if not ok:
        assert L.bsp_cache_compact(c, planes, stride, P16, 2, 4, P16, P16, P16, P16, None) == EINVAL


def test_lists_of_more_than_a_launch_are_refused(B, L):
    """Before anything is changed: extend has two kernels, the second with a workgroup for each entry."""
    c, s, n, out, want = cache(B), B._Strides(128, 64, 1), 1 << 24, ctypes.c_int64(), EUNSUPPORTED
    for m in (n, 2 ** 31 - 1):
        assert L.bsp_cache_append(c, m, P16, s, P16, s, P16, P16, P16, 1, 4, None, P16, None) == want
        assert L.bsp_cache_fork(2, 4, 10, P16, P16, P16, m, P16, P16, P16, None) == want
        assert L.bsp_cache_extend(c, 1, 0, P16, 2, 4, P16, P16, P16, m, P16, P16, P16, P16, None) == want
        assert L.bsp_cache_release(2, 4, 10, P16, P16, P16, m, P16, None) == want
        assert L.bsp_cache_scratch(c, 2, 4, m, ctypes.addressof(out)) == want
    assert L.bsp_cache_scratch(c, 2, 2 ** 31 - 1, n - 1, ctypes.addressof(out)) == 0 and out.value == 4 * (n - 1) << 31
