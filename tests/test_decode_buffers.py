"""Buffers that QuantLayer and PagedCache make: how long they live, and on whose stream they are."""

import weakref

import numpy as np
import pytest

from tests import decode_model as M


def test_an_outgrown_workspace_lives_on(monkeypatch):
    """CPU: a captured graph, or a call under way, may still write there."""
    import torch
    import paper_2111_11581_amd as B
    from paper_2111_11581_amd.layers import PagedCache
    monkeypatch.setattr(B, "_on_device", lambda **arrays: None)
    cache = PagedCache(1, 64, 512, 10, 16, 2, 64, device="cpu")
    seen, before = [], 0
    for batch in (1, 4, 4, 7, 64, 2):
        cache.reserve(batch, 8)
        assert cache.workspace.numel() >= B.bsp_attention_workspace(cache.shape, batch, 8, 512) > 0
        if cache.workspace.data_ptr() not in [p for p, _ in seen]:
            assert cache.workspace.numel() >= 2 * before
            before = cache.workspace.numel()
            seen.append((cache.workspace.data_ptr(), weakref.ref(cache.workspace)))
    assert len(seen) > 1 and all(w() is not None for _, w in seen)


def filled_cache(tokens, seqs=64, heads=8, kv=2, dim=64, seed=0):
    """A cache for 64 sequences, each of up to `tokens` tokens, in a table wide enough to be cut."""
    import torch
    from paper_2111_11581_amd.layers import PagedCache
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cache = PagedCache(1, seqs, 256, seqs * M.ceil(tokens, 16) + 1, 16, kv, dim)
    rows = torch.arange(seqs, dtype=torch.int32, device="cuda")
    pos = torch.empty_like(rows)
    cache.extend(rows, torch.full_like(rows, tokens) - rows, pos)
    cache.data.copy_(torch.randn(cache.data.shape, device="cuda", generator=gen))
    return cache, torch.randn(seqs, heads, dim, device="cuda", generator=gen).bfloat16()


@pytest.mark.gpu
def test_a_graph_after_a_larger_batch():
    """A step captured for 4 sequences, replayed after 64 had their attention and new arrays were made."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cache, q = filled_cache(300)
    rows = torch.arange(64, dtype=torch.int32, device="cuda")
    y, lse = torch.empty_like(q), torch.empty(64, 8, device="cuda")
    cache.reserve(4, 8)
    small = cache.workspace.numel()
    cache.attend(0, q[:4], y[:4], 0.125, rows[:4], lse=lse[:4])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(0, q[:4], y[:4], 0.125, rows[:4], lse=lse[:4])
    want, want_lse = torch.empty_like(y), torch.empty_like(lse)
    cache.attend(0, q, want, 0.125, rows, lse=want_lse)
    assert cache.workspace.numel() > small
    others = [torch.full((small,), 7, dtype=torch.uint8, device="cuda") for _ in range(20)]
    for _ in range(3):
        y.fill_(9)
        lse.fill_(9)
        graph.replay()
        cache.attend(0, q[4:], y[4:], 0.125, rows[4:], lse=lse[4:])
        torch.cuda.synchronize()
        assert torch.allclose(y.float(), want.float(), atol=2e-2) and torch.allclose(lse, want_lse, atol=1e-4)
        assert all(bool((o == 7).all()) for o in others)


@pytest.mark.gpu
@pytest.mark.parametrize("handle", [False, True])
def test_what_a_call_on_another_stream_makes(handle):
    """Memory that the current stream gave back while its own work there is still to come is not what a
    call on another stream writes its results to."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2111_11581_amd as B
    from paper_2111_11581_amd.layers import PackedLayer, QuantLayer
    rows, cols = 256, 512
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    w = torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    scheme = B.Scheme(rows, cols, 16, 32, B.COL, 4)
    quant, packed = QuantLayer(rows, cols, 64, B.F32, w), PackedLayer(scheme, B.F32, w)
    want = [quant.codes, quant.scales, quant.dequantize(), packed.mask, packed.tiles, packed.unpack()]
    torch.cuda.synchronize()
    left = [torch.empty(t.nbytes, dtype=torch.uint8, device="cuda") for t in want for _ in range(4)]
    torch.cuda._sleep(100_000_000)   # some 50 ms
    for t in left:
        t.fill_(0xA5)
    del left, t
    q, p = QuantLayer(rows, cols, 64, B.F32, w, stream=stream), PackedLayer(scheme, B.F32, w, stream=stream)
    got = [q.codes, q.scales, q.dequantize(stream=stream), p.mask, p.tiles, p.unpack(stream=stream)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
