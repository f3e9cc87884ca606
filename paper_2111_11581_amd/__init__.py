"""Block-structured pruned conv / FC inference on AMD MI355X (gfx950).

Thin ctypes binding of the C ABI in ``include/bsp.h`` (``libbsp.so``, built by
``python -m paper_2111_11581_amd.build``).  The functions below have the same
names as the C entry points and only marshal arguments: torch tensors supply
device pointers, torch's current HIP stream is the default stream.  Every step
of the computation runs in the library's HIP kernels; if the library is not
built, importing the functions raises - there is no fallback.
"""

from __future__ import annotations

import ctypes
import functools
import os

__all__ = [
    "F32", "BF16", "ROW", "COL", "UNSTRUCTURED", "DENSE", "PUNCHED", "ROWCOL", "PATTERN", "BspError", "Scheme", "ConvShape",
    "lib", "lib_path", "bsp_packed_sizes", "bsp_prune", "bsp_prune_noalloc", "bsp_pack", "bsp_unpack", "bsp_conv2d",
    "bsp_linear", "bsp_maxpool2x2", "bsp_status_string", "bsp_version", "bsp_to_bcs",
    "HEAD_MAJOR", "SLOT_MAJOR", "CacheShape", "bsp_q4_sizes", "bsp_q4_quantize", "bsp_q4_dequantize", "bsp_q4_linear",
    "bsp_attention_workspace", "bsp_attention", "bsp_cache_append", "bsp_cache_scratch", "bsp_cache_fork",
    "bsp_cache_extend", "bsp_cache_release", "bsp_cache_compact", "bsp_cache_copy",
]

_I64x4 = ctypes.c_int64 * 4
F32, BF16 = 0, 1
ROW, COL, UNSTRUCTURED, DENSE, PUNCHED, ROWCOL, PATTERN = 0, 1, 2, 3, 4, 5, 6

HEAD_MAJOR, SLOT_MAJOR = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "_build", "libbsp.so")
_lib = None


class BspError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {bsp_status_string(status)} ({status})")


class Scheme(ctypes.Structure):
    """bsp_scheme.  ``counts`` (optional) is a host int32 array of kept groups per
    block; set it with ``set_counts`` so that the array outlives the scheme's use."""
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "cols", "bh", "bw", "regularity", "rate", "khw")] + [
        ("counts", ctypes.POINTER(ctypes.c_int32))]

    def set_counts(self, counts):
        if counts is None:
            self._counts_buf = None
            self.counts = ctypes.POINTER(ctypes.c_int32)()
            return self
        flat = [int(v) for row in counts for v in (row if hasattr(row, "__iter__") else [row])]
        self._counts_buf = (ctypes.c_int32 * len(flat))(*flat)
        self.counts = ctypes.cast(self._counts_buf, ctypes.POINTER(ctypes.c_int32))
        return self


class ConvShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n", "cin", "h", "w", "kh", "kw", "stride_h",
                                               "stride_w", "pad_h", "pad_w")]


class CacheShape(ctypes.Structure):
    """bsp_cache: the pages of a cache's keys or values (one layer's)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "order", "pages", "page_size", "kv_heads", "head_dim")] + [
        ("page_stride", ctypes.c_int64)]

    @classmethod
    def of(cls, plane, order: int = HEAD_MAJOR) -> "CacheShape":
        """The shape of one plane of pages, [pages, kv_heads, page_size, head_dim] (HEAD_MAJOR) or
        [pages, page_size, kv_heads, head_dim] (SLOT_MAJOR), each page contiguous."""
        pages, a, b, dim = plane.shape
        heads, slots = (a, b) if order == HEAD_MAJOR else (b, a)
        code = next((c for c, t in _float_types().items() if t is plane.dtype), None)
        if code is None:
            raise ValueError(f"plane must be of fp32 or bf16, not {plane.dtype}")
        c = cls(code, order, pages, slots, heads, dim,
                plane.stride(0) if pages > 1 else 0)
        _plane_layout(bytes(c), "plane", plane.shape, plane.stride(), plane.dtype)
        _on_device(plane=plane)
        return c

    def plane_shape(self):
        inner = (self.kv_heads, self.page_size) if self.order == HEAD_MAJOR else (self.page_size, self.kv_heads)
        return (self.pages, *inner, self.head_dim)


class _Strides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("seq", "head", "dim")]


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load libbsp.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2111_11581_amd.build`")
    L = ctypes.CDLL(_LIB_PATH)
    P, I32, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_void_p
    sch, cs = P(Scheme), P(ConvShape)
    L.bsp_packed_sizes.argtypes = [sch, cs, I32, VP, VP, VP, VP]   # int64 results, by address
    L.bsp_prune.argtypes = [sch, I32, VP, VP, VP]
    L.bsp_prune_noalloc.argtypes = [sch, I32, VP, VP, VP]
    L.bsp_pack.argtypes = [sch, I32, VP, VP, VP, VP, VP, VP, cs, VP]
    L.bsp_unpack.argtypes = [sch, I32, VP, VP, VP, VP, VP]
    L.bsp_to_bcs.argtypes = [sch] + [VP] * 8
    L.bsp_conv2d.argtypes = [sch, cs, I32, I32, VP, VP, VP, I32, VP, VP]
    L.bsp_linear.argtypes = [sch, I32, I32, I32, VP, VP, VP, I32, VP, VP]
    L.bsp_maxpool2x2.argtypes = [I32, I32, I32, I32, I32, VP, VP, VP]
    L.bsp_status_string.argtypes = [I32]
    L.bsp_status_string.restype = ctypes.c_char_p
    L.bsp_version.argtypes = []
    I64, ca, sd = ctypes.c_int64, P(CacheShape), P(_Strides)
    L.bsp_q4_sizes.argtypes = [I32, I32, I32, VP, VP]
    L.bsp_q4_quantize.argtypes = [I32, I32, I32, I32, VP, VP, VP, VP, VP]
    L.bsp_q4_dequantize.argtypes = [I32, I32, I32, I32, VP, VP, VP, VP]
    L.bsp_q4_linear.argtypes = [I32] * 6 + [VP, VP, VP, VP, I32, VP, VP]
    L.bsp_cache_append.argtypes = [ca, I32, VP, sd, VP, sd, VP, VP, VP, I32, I32, VP, VP, VP]
    L.bsp_attention_workspace.argtypes = [ca, I32, I32, I32, VP]
    L.bsp_attention.argtypes = [ca, I32, I32, VP, sd, VP, VP, VP, I32, I32, VP, VP, ctypes.c_float, I32, VP, sd, VP, VP, VP]
    L.bsp_cache_scratch.argtypes = [ca, I32, I32, I32, VP]
    L.bsp_cache_fork.argtypes = [I32, I32, I32, VP, VP, VP, I32, VP, VP, VP, VP]
    L.bsp_cache_extend.argtypes = [ca, I32, I64, VP, I32, I32, VP, VP, VP, I32, VP, VP, VP, VP, VP]
    L.bsp_cache_release.argtypes = [I32, I32, I32, VP, VP, VP, I32, VP, VP]
    L.bsp_cache_compact.argtypes = [ca, I32, I64, VP, I32, I32, VP, VP, VP, VP, VP]
    L.bsp_cache_copy.argtypes = [ca, I32, I64, VP, I32, VP, VP, VP]
    for f in ("bsp_packed_sizes", "bsp_prune", "bsp_prune_noalloc", "bsp_pack", "bsp_unpack", "bsp_conv2d",
              "bsp_linear", "bsp_maxpool2x2", "bsp_version", "bsp_to_bcs", "bsp_q4_sizes", "bsp_q4_quantize",
              "bsp_q4_dequantize", "bsp_q4_linear", "bsp_cache_append", "bsp_attention_workspace", "bsp_attention",
              "bsp_cache_scratch", "bsp_cache_fork", "bsp_cache_extend", "bsp_cache_release", "bsp_cache_compact",
              "bsp_cache_copy"):
        getattr(L, f).restype = I32
    _lib = L
    return L


def _scheme(s) -> Scheme:
    if isinstance(s, Scheme):
        return s
    out = Scheme(int(s.rows), int(s.cols), int(s.bh), int(s.bw), int(s.regularity), int(s.rate),
                 int(getattr(s, "khw", 1)))
    return out.set_counts(getattr(s, "counts", None))


def _shape(c) -> ConvShape | None:
    if c is None or isinstance(c, ConvShape):
        return c
    return ConvShape(*[int(v) for v in c])


def _p(t):
    return None if t is None else t.data_ptr()


_raw_stream = None   # () -> handle of torch's current stream on the current device


def _raw_stream_getter():
    """torch.cuda.current_stream() builds a Stream object (3 us a call); the raw handle is
    the same value without it (0.3 us), where this torch offers it."""
    import torch
    torch.cuda.current_stream()   # initialises the device
    get, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if get is None or dev is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: get(dev())


def _stream(stream):
    global _raw_stream
    if stream is not None:
        return ctypes.c_void_p(int(getattr(stream, "cuda_stream", stream)))
    if _raw_stream is None:
        _raw_stream = _raw_stream_getter()
    return _raw_stream()


def _check(fn: str, st: int):
    if st != 0:
        raise BspError(fn, st)


def _need(name: str, t, nbytes: int):
    if t is None:
        raise ValueError(f"{name} is required")
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise ValueError(f"{name} holds {have} bytes, {nbytes} needed")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def bsp_status_string(status: int) -> str:
    return lib().bsp_status_string(int(status)).decode()


def bsp_version() -> int:
    return int(lib().bsp_version())


def bsp_packed_sizes(scheme, conv, wdt: int):
    """-> (n_values, n_indices, n_rowptr, dev_tile_bytes)."""
    out = _I64x4()
    sh = _shape(conv)
    a = ctypes.addressof(out)
    _check("bsp_packed_sizes", lib().bsp_packed_sizes(
        ctypes.byref(_scheme(scheme)), ctypes.byref(sh) if sh is not None else None, int(wdt), a, a + 8, a + 16, a + 24))
    return tuple(out)


def _esize(dt: int) -> int:
    return 4 if dt == F32 else 2


def bsp_prune(scheme, wdt: int, w, mask, stream=None):
    s = _scheme(scheme)
    _need("w", w, s.rows * s.cols * _esize(wdt))
    _need("mask", mask, s.rows * s.cols)
    _check("bsp_prune", lib().bsp_prune(ctypes.byref(s), int(wdt), _p(w), _p(mask), _stream(stream)))


def bsp_prune_noalloc(scheme, wdt: int, w, mask, stream=None):
    s = _scheme(scheme)
    _need("w", w, s.rows * s.cols * _esize(wdt))
    _need("mask", mask, s.rows * s.cols)
    _check("bsp_prune_noalloc", lib().bsp_prune_noalloc(ctypes.byref(s), int(wdt), _p(w), _p(mask),
                                                        _stream(stream)))


def bsp_pack(scheme, wdt: int, w, mask, values, indices, rowptr, dev_tiles, conv=None, stream=None):
    s = _scheme(scheme)
    nv, ni, nr, nb = bsp_packed_sizes(s, conv, wdt)
    _need("w", w, s.rows * s.cols * _esize(wdt))
    _need("mask", mask, s.rows * s.cols)
    _need("values", values, nv * _esize(wdt))
    if ni:
        _need("indices", indices, ni * 4)
    if nr:
        _need("rowptr", rowptr, nr * 4)
    _need("dev_tiles", dev_tiles, nb)
    sh = _shape(conv)
    _check("bsp_pack", lib().bsp_pack(ctypes.byref(s), int(wdt), _p(w), _p(mask), _p(values),
                                      _p(indices), _p(rowptr), _p(dev_tiles),
                                      ctypes.byref(sh) if sh is not None else None, _stream(stream)))


def bsp_unpack(scheme, wdt: int, values, indices, rowptr, w_out, stream=None):
    s = _scheme(scheme)
    _need("w_out", w_out, s.rows * s.cols * _esize(wdt))
    _check("bsp_unpack", lib().bsp_unpack(ctypes.byref(s), int(wdt), _p(values), _p(indices),
                                          _p(rowptr), _p(w_out), _stream(stream)))


def bsp_to_bcs(scheme, indices, rowptr, occurrence, compact_cols, col_stride, row_offset, n_runs, stream=None):
    s = _scheme(scheme)
    _need("row_offset", row_offset, (s.rows + 1) * 4)
    _need("n_runs", n_runs, 4)
    _check("bsp_to_bcs", lib().bsp_to_bcs(ctypes.byref(s), _p(indices), _p(rowptr), _p(occurrence),
                                          _p(compact_cols), _p(col_stride), _p(row_offset), _p(n_runs),
                                          _stream(stream)))


def bsp_conv2d(scheme, shape, in_dt: int, out_dt: int, x, dev_tiles, bias, relu: bool, y, stream=None):
    s, sh = _scheme(scheme), _shape(shape)
    ho = (sh.h + 2 * sh.pad_h - sh.kh) // sh.stride_h + 1
    wo = (sh.w + 2 * sh.pad_w - sh.kw) // sh.stride_w + 1
    _need("x", x, sh.n * sh.cin * sh.h * sh.w * _esize(in_dt))
    _need("y", y, sh.n * s.rows * ho * wo * _esize(out_dt))
    _need("dev_tiles", dev_tiles, bsp_packed_sizes(s, sh, in_dt)[3])
    if bias is not None:
        _need("bias", bias, s.rows * 4)
    _check("bsp_conv2d", lib().bsp_conv2d(ctypes.byref(s), ctypes.byref(sh), int(in_dt), int(out_dt),
                                          _p(x), _p(dev_tiles), _p(bias), int(bool(relu)), _p(y),
                                          _stream(stream)))


def bsp_linear(scheme, batch: int, in_dt: int, out_dt: int, x, dev_tiles, bias, relu: bool, y,
               stream=None):
    s = _scheme(scheme)
    _need("x", x, s.cols * batch * _esize(in_dt))
    _need("y", y, s.rows * batch * _esize(out_dt))
    _need("dev_tiles", dev_tiles, bsp_packed_sizes(s, None, in_dt)[3])
    if bias is not None:
        _need("bias", bias, s.rows * 4)
    _check("bsp_linear", lib().bsp_linear(ctypes.byref(s), int(batch), int(in_dt), int(out_dt), _p(x),
                                          _p(dev_tiles), _p(bias), int(bool(relu)), _p(y),
                                          _stream(stream)))


def bsp_maxpool2x2(dt: int, n: int, c: int, h: int, w: int, x, y, stream=None):
    _need("x", x, n * c * h * w * _esize(dt))
    _need("y", y, n * c * (h // 2) * (w // 2) * _esize(dt))
    _check("bsp_maxpool2x2", lib().bsp_maxpool2x2(int(dt), int(n), int(c), int(h), int(w), _p(x),
                                                  _p(y), _stream(stream)))


# ---- decode: 4-bit FC layers, attention over a paged cache, care of its pages ----
# What a call asks of the layout of its arrays is worked out once per layout and remembered (nothing
# else of an array is): an attention call is issued in 6.9 us so, in 10.4 us otherwise, and a short
# sequence's kernel takes no longer.

_int32 = None


_types = {}   # torch's types by their codes


def _float_types():
    if not _types:
        import torch
        _types.update({F32: torch.float32, BF16: torch.bfloat16})
    return _types


def _dev(name: str, t, nbytes: int, dt=None):
    """A contiguous device array of at least `nbytes`; not of another floating-point type than dt
    (bits in arrays of integers are taken as they are)."""
    if t is None or t.nbytes < nbytes or not t.is_contiguous():
        _need(name, t, nbytes)
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the device")
    if dt is not None and t.dtype is not _types.get(dt) and t.dtype is not _float_types().get(dt) and t.is_floating_point():
        raise ValueError(f"{name} must be of the type that the call names, not {t.dtype}")


def _ints(name: str, t, n: int):
    """A contiguous device array of at least n int32."""
    global _int32
    if _int32 is None:
        import torch
        _int32 = torch.int32
    if t is None or t.dtype is not _int32 or not t.is_cuda or not t.is_contiguous() or t.numel() < n:
        _dev(name, t, 4 * n)
        raise ValueError(f"{name} must be int32")


def _on_device(**arrays):
    for name, t in arrays.items():
        if not t.is_cuda:
            raise ValueError(f"{name} must be on the device")


def _plane_layout(key: bytes, name: str, shape, strides, dtype):
    """Keys or values of one layer: pages of the cache."""
    cache = CacheShape.from_buffer_copy(key)
    if tuple(shape) != cache.plane_shape() or dtype is not _float_types().get(cache.dtype):
        raise ValueError(f"{name} is not an array of the cache's pages")
    d = cache.head_dim
    page = cache.kv_heads * cache.page_size * d
    want = (cache.page_stride or page, (cache.page_size if cache.order == HEAD_MAJOR else cache.kv_heads) * d, d, 1)
    if any(n > 1 and have != s for n, have, s in zip(shape, strides, want)):
        raise ValueError(f"{name}: the pages are not contiguous, or not page_stride elements apart")


@functools.lru_cache(maxsize=4096)
def _layouts(key: bytes, names, n: int, heads: int, *arrays):
    """Strides of two [n, heads, head_dim] arrays of the cache's type; `arrays` are their, the keys'
    and the values' shape, strides and type."""
    cache = CacheShape.from_buffer_copy(key)
    out = []
    for name, shape, strides, dtype in zip(names, arrays[0::3], arrays[1::3], arrays[2::3]):
        if tuple(shape) != (n, heads, cache.head_dim) or dtype is not _float_types().get(cache.dtype):
            raise ValueError(f"{name} must be [{n}, {heads}, {cache.head_dim}] of the cache's type")
        out.append(_Strides(*strides))
    _plane_layout(key, "keys", *arrays[6:9])
    _plane_layout(key, "values", *arrays[9:])
    return out


def _table(table):
    if table.dim() != 2:
        raise ValueError("table must be [sequences, width]")
    _ints("table", table, 0)
    return table.shape


def bsp_q4_sizes(rows: int, cols: int, group: int):
    """-> (bytes of codes, elements of scales)."""
    out = (ctypes.c_int64 * 2)()
    a = ctypes.addressof(out)
    _check("bsp_q4_sizes", lib().bsp_q4_sizes(int(rows), int(cols), int(group), a, a + 8))
    return tuple(out)


_q4_sizes = functools.lru_cache(maxsize=4096)(bsp_q4_sizes)


def _q4_arrays(rows, cols, group, codes, scales):
    nc, ns = _q4_sizes(rows, cols, group)
    _dev("codes", codes, nc)
    _dev("scales", scales, ns * 2, BF16)


def bsp_q4_quantize(rows: int, cols: int, group: int, wdt: int, w, mask, codes, scales, stream=None):
    _q4_arrays(rows, cols, group, codes, scales)
    _dev("w", w, rows * cols * _esize(wdt), wdt)
    if mask is not None:
        _dev("mask", mask, rows * cols)
    _check("bsp_q4_quantize", lib().bsp_q4_quantize(rows, cols, group, wdt, _p(w), _p(mask), _p(codes), _p(scales),
                                                    _stream(stream)))


def bsp_q4_dequantize(rows: int, cols: int, group: int, wdt: int, codes, scales, w, stream=None):
    _q4_arrays(rows, cols, group, codes, scales)
    _dev("w", w, rows * cols * _esize(wdt), wdt)
    _check("bsp_q4_dequantize", lib().bsp_q4_dequantize(rows, cols, group, wdt, _p(codes), _p(scales), _p(w),
                                                        _stream(stream)))


def bsp_q4_linear(rows: int, cols: int, group: int, batch: int, in_dt: int, out_dt: int, x, codes, scales, bias,
                  relu: bool, y, stream=None):
    _q4_arrays(rows, cols, group, codes, scales)
    _dev("x", x, cols * batch * _esize(in_dt), in_dt)
    _dev("y", y, rows * batch * _esize(out_dt), out_dt)
    if bias is not None:
        _dev("bias", bias, rows * 4, F32)
    st = lib().bsp_q4_linear(rows, cols, group, batch, in_dt, out_dt, x.data_ptr(), codes.data_ptr(), scales.data_ptr(),
                             _p(bias), 1 if relu else 0, y.data_ptr(), _stream(stream))
    if st:
        raise BspError("bsp_q4_linear", st)


def bsp_cache_append(cache: CacheShape, k, v, keys, values, table, pos, rows=None, stream=None):
    """k and v: [tokens, kv_heads, head_dim] of any strides."""
    n, key = k.shape[0], bytes(cache)
    ks, vs = _layouts(key, ("k", "v"), n, cache.kv_heads, k.shape, k.stride(), k.dtype, v.shape, v.stride(), v.dtype,
                      keys.shape, keys.stride(), keys.dtype, values.shape, values.stride(), values.dtype)
    if not (k.is_cuda and v.is_cuda and keys.is_cuda and values.is_cuda):
        _on_device(k=k, v=v, keys=keys, values=values)
    seqs, width = _table(table)
    _ints("pos", pos, n)
    if rows is not None:
        _ints("rows", rows, n)
    st = lib().bsp_cache_append(cache, n, k.data_ptr(), ks, v.data_ptr(), vs, keys.data_ptr(), values.data_ptr(),
                                table.data_ptr(), seqs, width, _p(rows), pos.data_ptr(), _stream(stream))
    if st:
        raise BspError("bsp_cache_append", st)


def bsp_attention_workspace(cache: CacheShape, batch: int, heads: int, width: int) -> int:
    """Bytes of bsp_attention's workspace."""
    out = ctypes.c_int64()
    _check("bsp_attention_workspace", lib().bsp_attention_workspace(cache, int(batch), int(heads), int(width),
                                                                    ctypes.addressof(out)))
    return out.value


@functools.lru_cache(maxsize=4096)
def _workspace(key: bytes, batch: int, heads: int, width: int) -> int:
    return bsp_attention_workspace(CacheShape.from_buffer_copy(key), batch, heads, width)


def bsp_attention(cache: CacheShape, q, keys, values, table, lens, y, scale: float, window: int = 0, rows=None, lse=None,
                  workspace=None, stream=None):
    """q and y: [batch, heads, head_dim] of any strides (y's elements distinct)."""
    (batch, heads, _), key = q.shape, bytes(cache)
    qs, ys = _layouts(key, ("q", "y"), batch, heads, q.shape, q.stride(), q.dtype, y.shape, y.stride(), y.dtype,
                      keys.shape, keys.stride(), keys.dtype, values.shape, values.stride(), values.dtype)
    if not (q.is_cuda and y.is_cuda and keys.is_cuda and values.is_cuda):
        _on_device(q=q, y=y, keys=keys, values=values)
    seqs, width = _table(table)
    _ints("lens", lens, seqs)
    if rows is not None:
        _ints("rows", rows, batch)
    if lse is not None:
        _dev("lse", lse, batch * heads * 4, F32)
    need = _workspace(key, batch, heads, width)
    if need:
        _dev("workspace", workspace, need)
    st = lib().bsp_attention(cache, batch, heads, q.data_ptr(), qs, keys.data_ptr(), values.data_ptr(), table.data_ptr(),
                             seqs, width, _p(rows), lens.data_ptr(), scale, window, y.data_ptr(), ys, _p(lse),
                             _p(workspace), _stream(stream))
    if st:
        raise BspError("bsp_attention", st)


def bsp_cache_scratch(cache: CacheShape, seqs: int, width: int, n: int) -> int:
    """Bytes of the scratch of fork, extend and compact with lists of up to n sequences."""
    out = ctypes.c_int64()
    _check("bsp_cache_scratch", lib().bsp_cache_scratch(cache, int(seqs), int(width), int(n), ctypes.addressof(out)))
    return out.value


@functools.lru_cache(maxsize=4096)
def _scratch(key: bytes, seqs: int, width: int, n: int) -> int:
    return bsp_cache_scratch(CacheShape.from_buffer_copy(key), seqs, width, n)


def _state(table, lens, refs, pages: int):
    seqs, width = _table(table)
    _ints("lens", lens, seqs)
    _ints("refs", refs, pages)
    return seqs, width


@functools.lru_cache(maxsize=1024)
def _planes_layout(key: bytes, shape, strides, dtype):
    """Planes and plane stride of [planes, *plane_shape]."""
    if len(shape) != 5 or shape[0] < 1:
        raise ValueError("data must be [planes, pages, ., ., head_dim]")
    _plane_layout(key, "data", shape[1:], strides[1:], dtype)
    return shape[0], strides[0] if shape[0] > 1 else 0


def _planes(key: bytes, data):
    if not data.is_cuda:
        _on_device(data=data)
    return _planes_layout(key, data.shape, data.stride(), data.dtype)


def bsp_cache_fork(table, lens, refs, parents, children, scratch, stream=None):
    n, pages = parents.numel(), refs.numel()
    seqs, width = _state(table, lens, refs, pages)
    _ints("parents", parents, n)
    _ints("children", children, n)
    _dev("scratch", scratch, 4 * n * (width + 1))
    _check("bsp_cache_fork", lib().bsp_cache_fork(seqs, width, pages, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), n,
                                                  parents.data_ptr(), children.data_ptr(), scratch.data_ptr(),
                                                  _stream(stream)))


def bsp_cache_extend(cache: CacheShape, data, table, lens, refs, rows, counts, pos, scratch, stream=None):
    key, n = bytes(cache), rows.numel()
    planes, plane_stride = _planes(key, data)
    seqs, width = _state(table, lens, refs, cache.pages)
    _ints("rows", rows, n)
    _ints("counts", counts, n)
    _ints("pos", pos, n)
    _dev("scratch", scratch, _scratch(key, seqs, width, n))
    _check("bsp_cache_extend", lib().bsp_cache_extend(cache, planes, plane_stride, data.data_ptr(), seqs, width,
                                                      table.data_ptr(), lens.data_ptr(), refs.data_ptr(), n,
                                                      rows.data_ptr(), counts.data_ptr(), pos.data_ptr(),
                                                      scratch.data_ptr(), _stream(stream)))


def bsp_cache_release(table, lens, refs, rows, stream=None):
    n, pages = rows.numel(), refs.numel()
    seqs, width = _state(table, lens, refs, pages)
    _ints("rows", rows, n)
    _check("bsp_cache_release", lib().bsp_cache_release(seqs, width, pages, table.data_ptr(), lens.data_ptr(),
                                                        refs.data_ptr(), n, rows.data_ptr(), _stream(stream)))


def bsp_cache_compact(cache: CacheShape, data, table, refs, info, scratch, stream=None):
    key = bytes(cache)
    planes, plane_stride = _planes(key, data)
    seqs, width = _table(table)
    _ints("refs", refs, cache.pages)
    _ints("info", info, 2)
    _dev("scratch", scratch, _scratch(key, seqs, width, 0))
    _check("bsp_cache_compact", lib().bsp_cache_compact(cache, planes, plane_stride, data.data_ptr(), seqs, width,
                                                        table.data_ptr(), refs.data_ptr(), info.data_ptr(),
                                                        scratch.data_ptr(), _stream(stream)))


def bsp_cache_copy(cache: CacheShape, data, src, dst, stream=None):
    planes, plane_stride = _planes(bytes(cache), data)
    n = src.numel()
    _ints("src", src, n)
    _ints("dst", dst, n)
    _check("bsp_cache_copy", lib().bsp_cache_copy(cache, planes, plane_stride, data.data_ptr(), n, src.data_ptr(),
                                                  dst.data_ptr(), _stream(stream)))
