"""Convenience wrappers that allocate the library's buffers with torch.

Still argument marshalling only: pruning, packing and the forward run in the
HIP kernels behind the C ABI.
"""

from __future__ import annotations

import contextlib

import torch

from . import (BF16, F32, HEAD_MAJOR, CacheShape, ConvShape, Scheme, bsp_attention, bsp_attention_workspace,
               bsp_cache_append, bsp_cache_compact, bsp_cache_copy, bsp_cache_extend, bsp_cache_fork, bsp_cache_release,
               bsp_cache_scratch, bsp_conv2d, bsp_linear, bsp_pack, bsp_packed_sizes, bsp_prune, bsp_q4_dequantize,
               bsp_q4_linear, bsp_q4_quantize, bsp_q4_sizes, bsp_unpack)

TORCH_DT = {F32: torch.float32, BF16: torch.bfloat16}


def _made_on(stream, device):
    """Arrays that a call on ``stream`` writes are made on it: torch gives out memory that earlier work
    of its current stream may still be using, which only that stream's own later work waits for."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device)
    return torch.cuda.stream(stream)


class PackedLayer:
    """Pruned + packed weights of one conv (conv is a ConvShape) or FC (conv None) layer.

    ``w`` is the GEMM-form weight matrix on the device (rows x cols, fp32 or
    bf16).  ``mask`` may be given (it is then validated by bsp_pack);
    otherwise bsp_prune computes it.
    """

    def __init__(self, scheme, wdt: int, w: torch.Tensor, conv=None, mask: torch.Tensor | None = None,
                 stream=None):
        self.scheme = scheme if isinstance(scheme, Scheme) else Scheme(
            scheme.rows, scheme.cols, scheme.bh, scheme.bw, scheme.regularity, scheme.rate,
            getattr(scheme, "khw", 1)).set_counts(getattr(scheme, "counts", None))
        self.wdt = wdt
        self.conv = conv if (conv is None or isinstance(conv, ConvShape)) else ConvShape(*conv)
        dev = w.device
        R, C = self.scheme.rows, self.scheme.cols
        if mask is None:
            with _made_on(stream, dev):
                mask = torch.empty(R * C, dtype=torch.uint8, device=dev)
            bsp_prune(self.scheme, wdt, w, mask, stream)
        self.mask = mask
        nv, ni, nr, nb = bsp_packed_sizes(self.scheme, self.conv, wdt)
        with _made_on(stream, dev):
            self.values = torch.empty(max(nv, 1), dtype=TORCH_DT[wdt], device=dev)
            self.indices = torch.empty(max(ni, 1), dtype=torch.int32, device=dev)
            self.rowptr = torch.empty(max(nr, 1), dtype=torch.int32, device=dev)
            self.tiles = torch.empty(nb, dtype=torch.uint8, device=dev)
        self.n_values, self.n_indices, self.n_rowptr = nv, ni, nr
        bsp_pack(self.scheme, wdt, w, mask, self.values, self.indices, self.rowptr, self.tiles,
                 self.conv, stream)

    def unpack(self, stream=None) -> torch.Tensor:
        R, C = self.scheme.rows, self.scheme.cols
        with _made_on(stream, self.tiles.device):
            out = torch.empty(R * C, dtype=TORCH_DT[self.wdt], device=self.tiles.device)
        bsp_unpack(self.scheme, self.wdt, self.values, self.indices, self.rowptr, out, stream)
        return out

    def conv2d(self, x, y, n: int, out_dt: int, bias=None, relu=False, stream=None):
        c = self.conv
        shape = ConvShape(n, c.cin, c.h, c.w, c.kh, c.kw, c.stride_h, c.stride_w, c.pad_h, c.pad_w)
        bsp_conv2d(self.scheme, shape, self.wdt, out_dt, x, self.tiles, bias, relu, y, stream)

    def linear(self, x, y, batch: int, out_dt: int, bias=None, relu=False, stream=None):
        bsp_linear(self.scheme, batch, self.wdt, out_dt, x, self.tiles, bias, relu, y, stream)


class QuantLayer:
    """4-bit weights of an FC layer: ``w`` (rows x cols, fp32 or bf16, on the device) in groups of
    ``group`` columns.  Weights that ``mask`` (as from bsp_prune) removes are exactly 0."""

    def __init__(self, rows: int, cols: int, group: int, wdt: int, w: torch.Tensor, mask: torch.Tensor | None = None,
                 stream=None):
        self.rows, self.cols, self.group = rows, cols, group
        nc, ns = bsp_q4_sizes(rows, cols, group)
        with _made_on(stream, w.device):
            self.codes = torch.empty(nc, dtype=torch.uint8, device=w.device)
            self.scales = torch.empty(ns, dtype=torch.bfloat16, device=w.device)
        bsp_q4_quantize(rows, cols, group, wdt, w, mask, self.codes, self.scales, stream)

    def dequantize(self, wdt: int = F32, stream=None) -> torch.Tensor:
        with _made_on(stream, self.codes.device):
            out = torch.empty(self.rows, self.cols, dtype=TORCH_DT[wdt], device=self.codes.device)
        bsp_q4_dequantize(self.rows, self.cols, self.group, wdt, self.codes, self.scales, out, stream)
        return out

    def linear(self, x, y, batch: int, in_dt: int, out_dt: int, bias=None, relu=False, stream=None):
        bsp_q4_linear(self.rows, self.cols, self.group, batch, in_dt, out_dt, x, self.codes, self.scales, bias, relu, y,
                      stream)


class PagedCache:
    """Keys and values of ``layers`` layers for up to ``seqs`` sequences of up to ``width`` pages, in
    ``pages`` pages.  ``longest`` is the longest list that a call takes.

    Tables, lengths and counts are on the device and are never read by the host; lists are int32
    tensors on the device.  The scratch is the cache's own, so its calls belong on one stream (or on
    streams that wait for each other); it is made on torch's current stream.
    """

    def __init__(self, layers: int, seqs: int, width: int, pages: int, page_size: int, kv_heads: int, head_dim: int,
                 dtype: int = BF16, order: int = HEAD_MAJOR, longest: int | None = None, device="cuda"):
        inner = (kv_heads, page_size) if order == HEAD_MAJOR else (page_size, kv_heads)
        self.data = torch.zeros(2 * layers, pages, *inner, head_dim, dtype=TORCH_DT[dtype], device=device)
        self.shape = CacheShape.of(self.data[0], order)
        self.planes = [(self.data[2 * i], self.data[2 * i + 1]) for i in range(layers)]
        self.table = torch.full((seqs, width), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)
        self.info = torch.zeros(2, dtype=torch.int32, device=device)
        n = seqs if longest is None else longest
        self.scratch = torch.empty(bsp_cache_scratch(self.shape, seqs, width, n), dtype=torch.uint8, device=device)
        self.workspace = torch.empty(0, dtype=torch.uint8, device=device)
        self._outgrown = []

    def extend(self, rows, counts, pos, stream=None):
        """Room for counts[i] more tokens in sequence rows[i]; pos receives where they begin, or -1."""
        bsp_cache_extend(self.shape, self.data, self.table, self.lens, self.refs, rows, counts, pos, self.scratch, stream)

    def append(self, layer: int, k, v, pos, rows=None, stream=None):
        keys, values = self.planes[layer]
        bsp_cache_append(self.shape, k, v, keys, values, self.table, pos, rows, stream)

    def reserve(self, batch: int, heads: int, stream=None):
        """A workspace for attend with `batch` sequences; attend makes one where this was not called.
        Captured graphs and calls under way hold the one they were given, so that it lives as long as
        the cache does; each is at least twice the one before, and all before take no more than it."""
        need = bsp_attention_workspace(self.shape, batch, heads, self.table.shape[1])
        if self.workspace.numel() < need:
            self._outgrown.append(self.workspace)
            need = max(need, 2 * self.workspace.numel())
            with _made_on(stream, self.table.device):
                self.workspace = torch.empty(need, dtype=torch.uint8, device=self.table.device)

    def attend(self, layer: int, q, y, scale: float, rows=None, window: int = 0, lse=None, stream=None):
        """Attention of one token of each sequence rows[i] over what its pages hold."""
        self.reserve(q.shape[0], q.shape[1], stream)
        keys, values = self.planes[layer]
        bsp_attention(self.shape, q, keys, values, self.table, self.lens, y, scale, window, rows, lse, self.workspace, stream)

    def fork(self, parents, children, stream=None):
        bsp_cache_fork(self.table, self.lens, self.refs, parents, children, self.scratch, stream)

    def release(self, rows, stream=None):
        bsp_cache_release(self.table, self.lens, self.refs, rows, stream)

    def compact(self, stream=None):
        """Moves the pages in use to the front; -> (pages in use, pages moved) on the device."""
        bsp_cache_compact(self.shape, self.data, self.table, self.refs, self.info, self.scratch, stream)
        return self.info

    def copy(self, src, dst, stream=None):
        bsp_cache_copy(self.shape, self.data, src, dst, stream)
