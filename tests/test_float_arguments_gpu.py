"""Calls refuse arrays of another type where they take float32."""

import pytest

from tests.test_sample_gpu import B   # noqa: F401 (a fixture, which loads torch first)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["int32", "int64", "uint8", "float64"])
def test_calls(B, dtype):
    import torch
    bad = torch.ones(4096, dtype=getattr(torch, dtype), device="cuda")
    f, i = torch.ones(64, device="cuda"), torch.ones(64, dtype=torch.int32, device="cuda")
    names = []

    def refused(name, call):
        with pytest.raises(ValueError, match=f"^{name} must be"):
            call({name: bad})
        names.append(name)
    good = dict(u=f, temperature=f, top_p=f, min_p=f, logp=f)
    for name in good:
        refused(name, lambda kw: B.bsp_sample(B.F32, torch.zeros(4, 50, device="cuda"), tokens=i, **{**good, **kw}))
    rope, freqs = B.Rope(B.ROPE_HALF, 8), torch.zeros(4, dtype=torch.float64, device="cuda")
    x = torch.zeros(2, 2, 8, device="cuda")
    refused("norm", lambda kw: B.bsp_rotary(B.F32, rope, freqs, x, i, x, **kw))
    data = torch.zeros(2, 2, 2, 4, 8, device="cuda")
    cache, table = B.CacheShape.of(data[0]), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    for name in ("q_norm", "k_norm"):
        refused(name, lambda kw: B.bsp_cache_append_rotary(cache, rope, freqs, x, x, x, x, *data, table, i, **kw))
    refused("lse", lambda kw: B.bsp_attention_prefix(cache, x, *data, table, i, i, i[:1], x, 1.0, **kw))
    assert len(names) == 9
