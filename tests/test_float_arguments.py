"""Named arrays of float32 are refused where they are of another type, whose bits would be read as numbers."""

import pytest

from tests.test_decode_abi import B   # noqa: F401 (a fixture)


def test_types(B):
    import torch

    class OnDevice(torch.Tensor):   # what the check looks at says so
        is_cuda = True

    def array(dtype, n=4):
        return torch.zeros(n, dtype=dtype).as_subclass(OnDevice)
    B._floats("u", array(torch.float32), 4)
    for dtype in (torch.int32, torch.int64, torch.uint8, torch.bool, torch.float64, torch.float16, torch.bfloat16):
        with pytest.raises(ValueError):
            B._floats("u", array(dtype, 16), 4)
    for dtype in (torch.int32, torch.int64, torch.uint8):
        with pytest.raises(ValueError, match="u must be float32"):
            B._floats("u", array(dtype, 16), 4)
    with pytest.raises(ValueError, match="12 bytes"):
        B._floats("u", array(torch.float32, 3), 4)
    with pytest.raises(ValueError, match="contiguous"):
        B._floats("u", array(torch.float32, 8)[::2], 4)
    with pytest.raises(ValueError, match="device"):
        B._floats("u", torch.zeros(4), 4)
    with pytest.raises(ValueError, match="required"):
        B._floats("u", None, 4)
