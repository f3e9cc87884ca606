"""Limits of the decode operators: sizes, alignment, layouts and types at which a call has to be refused
or to ask for more.  CPU only: no call here launches a kernel."""

import ctypes

import pytest

from tests.test_decode_abi import EINVAL, P16, B, L, cache   # noqa: F401 (B and L are fixtures)


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
