// C ABI entry points of the decode operators: argument validation and dispatch.  Nothing is kept
// between calls; every device buffer belongs to the caller.
#include <climits>

#include <hip/hip_runtime.h>

#include "bsp_decode.h"

using namespace bsp;

namespace {

inline hipStream_t S(void *stream) { return (hipStream_t)stream; }
inline bsp_status status(hipError_t e) { return e == hipSuccess ? BSP_OK : BSP_EDEVICE; }
inline bool dtype_ok(int dt) { return dt == BSP_F32 || dt == BSP_BF16; }
inline int esize(int dt) { return dt == BSP_F32 ? 4 : 2; }
inline bool aligned(const void *p, int bytes) { return (uintptr_t)p % bytes == 0; }

bool q4_ok(int32_t rows, int32_t cols, int32_t group) {
    return rows >= 1 && rows <= INT32_MAX - 15 && cols >= 1 && (group == 32 || group == 64 || group == 128);
}

// One launch covers the matrix in tiles of 16 x 128.
bool q4_fits(const Q4Shape &s) { return (int64_t)s.rows16 / 16 * ((s.stride + 63) / 64) < 1 << 24; }

bsp_status check_cache(const bsp_cache *c) {
    if (!c || !dtype_ok(c->dtype) || (c->order != BSP_HEAD_MAJOR && c->order != BSP_SLOT_MAJOR)) return BSP_EINVAL;
    if (c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return BSP_EINVAL;
    if (c->head_dim % 8 || c->head_dim > 256) return BSP_EUNSUPPORTED;
    // of page_size and kv_heads, neither product with head_dim passes 32 bits
    if ((int64_t)c->page_size * c->kv_heads > INT32_MAX / 256) return BSP_EUNSUPPORTED;
    if (c->page_stride) {
        if (c->page_stride < (int64_t)c->page_size * c->kv_heads * c->head_dim) return BSP_EINVAL;
        if (c->page_stride > INT64_MAX / 8 / c->pages || c->page_stride % (16 / esize(c->dtype))) return BSP_EINVAL;
    }
    return BSP_OK;
}

constexpr int64_t kMaxTokens = 1 << 30;   // of a sequence: 32-bit numbers count positions, with room to round up

bsp_status check_table(const int32_t *table, int32_t seqs, int32_t width, int32_t page_size) {
    if (seqs < 0 || width < 0 || (!table && (int64_t)seqs * width > 0)) return BSP_EINVAL;
    return (int64_t)width * page_size > kMaxTokens ? BSP_EUNSUPPORTED : BSP_OK;
}

constexpr int32_t kMostListed = (1 << 24) - 1;   // a workgroup of 256 for each: a launch has fewer than 2^32 threads

bsp_status check_pages(const int32_t *table, const int32_t *lens, const int32_t *refs, int32_t seqs, int32_t width,
                       int32_t pages, int32_t n) {
    if (seqs < 0 || width < 0 || pages < 1 || n < 0 || !refs) return BSP_EINVAL;
    if ((!table && (int64_t)seqs * width > 0) || (!lens && seqs > 0)) return BSP_EINVAL;
    return n > kMostListed ? BSP_EUNSUPPORTED : BSP_OK;
}

bsp_status check_planes(const bsp_cache *c, int32_t planes, int64_t plane_stride, const void *data) {
    if (const bsp_status st = check_cache(c); st != BSP_OK) return st;
    if (!data || planes < 0 || plane_stride < 0 || !aligned(data, 16)) return BSP_EINVAL;
    if (plane_stride % (16 / esize(c->dtype)) || plane_stride > INT64_MAX / 8 / std::max(planes, 1)) return BSP_EINVAL;
    if (planes < 2) return BSP_OK;
    // no overlap: plane after plane, or the planes' pages side by side within a page's stride
    const int64_t page = (int64_t)c->page_size * c->kv_heads * c->head_dim, stride = c->page_stride ? c->page_stride : page;
    const bool after = plane_stride >= (c->pages - 1) * stride + page;
    const bool beside = plane_stride >= page && (planes - 1) * plane_stride + page <= stride;
    return after || beside ? BSP_OK : BSP_EINVAL;
}

PlanesArgs planes_args(const bsp_cache *c, int32_t planes, int64_t plane_stride, void *data) {
    PlanesArgs d;
    d.c = cache_args(*c), d.planes = planes, d.plane_stride = plane_stride, d.data = data;
    return d;
}

}  // namespace

extern "C" {

bsp_status bsp_q4_sizes(int32_t rows, int32_t cols, int32_t group, int64_t *code_bytes, int64_t *n_scales) {
    if (!code_bytes || !n_scales || !q4_ok(rows, cols, group)) return BSP_EINVAL;
    const Q4Shape s = q4_shape(rows, cols, group);
    *code_bytes = s.rows * s.stride;
    *n_scales = (int64_t)s.n_groups * s.rows16;
    return BSP_OK;
}

bsp_status bsp_q4_quantize(int32_t rows, int32_t cols, int32_t group, bsp_dtype wdt, const void *w, const uint8_t *mask,
                           uint8_t *codes, void *scales, void *stream) {
    if (!q4_ok(rows, cols, group) || !dtype_ok(wdt) || !w || !codes || !scales) return BSP_EINVAL;
    if (!aligned(codes, 16) || !aligned(scales, 8) || !aligned(w, esize(wdt))) return BSP_EINVAL;
    const Q4Shape s = q4_shape(rows, cols, group);
    if (!q4_fits(s)) return BSP_EUNSUPPORTED;
    return status(launch_q4_quantize(s, wdt, w, mask, codes, (uint16_t *)scales, S(stream)));
}

bsp_status bsp_q4_dequantize(int32_t rows, int32_t cols, int32_t group, bsp_dtype wdt, const uint8_t *codes,
                             const void *scales, void *w, void *stream) {
    if (!q4_ok(rows, cols, group) || !dtype_ok(wdt) || !w || !codes || !scales) return BSP_EINVAL;
    if (!aligned(codes, 16) || !aligned(scales, 8) || !aligned(w, esize(wdt))) return BSP_EINVAL;
    const Q4Shape s = q4_shape(rows, cols, group);
    if (!q4_fits(s)) return BSP_EUNSUPPORTED;
    return status(launch_q4_dequantize(s, wdt, codes, (const uint16_t *)scales, w, S(stream)));
}

bsp_status bsp_q4_linear(int32_t rows, int32_t cols, int32_t group, int32_t batch, bsp_dtype in_dt, bsp_dtype out_dt,
                         const void *x, const uint8_t *codes, const void *scales, const float *bias, int32_t relu, void *y,
                         void *stream) {
    if (!q4_ok(rows, cols, group) || !dtype_ok(in_dt) || !dtype_ok(out_dt) || batch < 0) return BSP_EINVAL;
    if (!codes || !scales || !aligned(codes, 16) || !aligned(scales, 8) || (batch > 0 && (!x || !y))) return BSP_EINVAL;
    if (!aligned(x, esize(in_dt)) || !aligned(y, esize(out_dt)) || !aligned(bias, 4)) return BSP_EINVAL;
    // offsets in x, and in the codes of 64 rows, are 32-bit numbers of bytes
    if ((int64_t)cols * batch > (int64_t)UINT32_MAX / esize(in_dt) || (int64_t)cols * batch > INT32_MAX) return BSP_EUNSUPPORTED;
    if ((int64_t)rows * batch > INT32_MAX || cols > 1 << 26 || rows > 1 << 26) return BSP_EUNSUPPORTED;
    if (batch > 1 << 19) return BSP_EUNSUPPORTED;   // tiles of 16 vectors are a grid's y
    if (batch == 0) return BSP_OK;
    return status(launch_q4_linear(q4_shape(rows, cols, group), batch, in_dt, out_dt, x, codes, (const uint16_t *)scales,
                                   bias, relu ? 1 : 0, y, S(stream)));
}

bsp_status bsp_cache_append(const bsp_cache *cache, int32_t n, const void *k, const bsp_strides *ks, const void *v,
                            const bsp_strides *vs, void *keys, void *values, const int32_t *table, int32_t seqs,
                            int32_t width, const int32_t *rows, const int32_t *pos, void *stream) {
    if (const bsp_status st = check_cache(cache); st != BSP_OK) return st;
    if (n < 0 || !ks || !vs || !keys || !values || !aligned(keys, 16) || !aligned(values, 16)) return BSP_EINVAL;
    if (n > 0 && (!k || !v || !pos)) return BSP_EINVAL;
    if (!aligned(k, esize(cache->dtype)) || !aligned(v, esize(cache->dtype))) return BSP_EINVAL;
    if (const bsp_status st = check_table(table, seqs, width, cache->page_size); st != BSP_OK) return st;
    if (n > kMostListed) return BSP_EUNSUPPORTED;
    if (n == 0 || (int64_t)seqs * width == 0) return BSP_OK;
    AppendArgs a;
    a.c = cache_args(*cache);
    a.k = k, a.v = v, a.keys = keys, a.values = values, a.ks = *ks, a.vs = *vs;
    a.table = table, a.rows = rows, a.pos = pos, a.n = n, a.seqs = seqs, a.width = width;
    return status(launch_append(a, S(stream)));
}

bsp_status bsp_attention_workspace(const bsp_cache *cache, int32_t batch, int32_t heads, int32_t width, int64_t *bytes) {
    if (const bsp_status st = check_cache(cache); st != BSP_OK) return st;
    if (!bytes || batch < 0 || heads < 1 || heads % cache->kv_heads || width < 0) return BSP_EINVAL;
    if ((int64_t)width * cache->page_size > kMaxTokens || (int64_t)batch * heads > INT32_MAX / 256) return BSP_EUNSUPPORTED;
    *bytes = attention_workspace(cache_args(*cache), batch, heads, width);
    return BSP_OK;
}

bsp_status bsp_attention(const bsp_cache *cache, int32_t batch, int32_t heads, const void *q, const bsp_strides *qs,
                         const void *keys, const void *values, const int32_t *table, int32_t seqs, int32_t width,
                         const int32_t *rows, const int32_t *lens, float scale, int32_t window, void *y,
                         const bsp_strides *ys, float *lse, void *workspace, void *stream) {
    if (const bsp_status st = check_cache(cache); st != BSP_OK) return st;
    if (batch < 0 || heads < 1 || heads % cache->kv_heads || window < 0 || !qs || !ys) return BSP_EINVAL;
    if (!keys || !values || !aligned(keys, 16) || !aligned(values, 16)) return BSP_EINVAL;
    if (batch > 0 && (!q || !y || (!lens && seqs > 0))) return BSP_EINVAL;
    if (!aligned(q, esize(cache->dtype)) || !aligned(y, esize(cache->dtype)) || !aligned(lse, 4)) return BSP_EINVAL;
    if (const bsp_status st = check_table(table, seqs, width, cache->page_size); st != BSP_OK) return st;
    if ((int64_t)batch * heads > INT32_MAX / 256) return BSP_EUNSUPPORTED;
    if (batch == 0) return BSP_OK;
    AttnArgs a;
    a.c = cache_args(*cache);
    if (attention_workspace(a.c, batch, heads, width) > 0 && (!workspace || !aligned(workspace, 16))) return BSP_EINVAL;
    a.q = q, a.keys = keys, a.values = values, a.y = y, a.lse = lse, a.qs = *qs, a.ys = *ys;
    a.table = table, a.rows = rows, a.lens = lens, a.batch = batch, a.heads = heads;
    a.group = heads / cache->kv_heads, a.seqs = seqs, a.width = width, a.window = window, a.scale = scale;
    a.workspace = workspace;
    return status(launch_attention(a, S(stream)));
}

bsp_status bsp_cache_scratch(const bsp_cache *cache, int32_t seqs, int32_t width, int32_t n, int64_t *bytes) {
    if (const bsp_status st = check_cache(cache); st != BSP_OK) return st;
    if (!bytes || seqs < 0 || width < 0 || n < 0) return BSP_EINVAL;
    if (n > kMostListed) return BSP_EUNSUPPORTED;
    *bytes = pages_scratch(cache->pages, width, n);
    return BSP_OK;
}

bsp_status bsp_cache_fork(int32_t seqs, int32_t width, int32_t pages, int32_t *table, int32_t *lens, int32_t *refs,
                          int32_t n, const int32_t *parents, const int32_t *children, void *scratch, void *stream) {
    if (const bsp_status st = check_pages(table, lens, refs, seqs, width, pages, n); st != BSP_OK) return st;
    if (n > 0 && (!parents || !children || !scratch || !aligned(scratch, 16))) return BSP_EINVAL;
    if (n == 0 || seqs == 0) return BSP_OK;
    return status(launch_fork({seqs, width, pages, table, lens, refs, n, (int32_t *)scratch}, parents, children, S(stream)));
}

bsp_status bsp_cache_extend(const bsp_cache *cache, int32_t planes, int64_t plane_stride, void *data, int32_t seqs,
                            int32_t width, int32_t *table, int32_t *lens, int32_t *refs, int32_t n, const int32_t *rows,
                            const int32_t *counts, int32_t *pos, void *scratch, void *stream) {
    if (const bsp_status st = check_planes(cache, planes, plane_stride, data); st != BSP_OK) return st;
    if (const bsp_status st = check_pages(table, lens, refs, seqs, width, cache->pages, n); st != BSP_OK) return st;
    if (n > 0 && (!rows || !counts || !pos || !scratch || !aligned(scratch, 16))) return BSP_EINVAL;
    if ((int64_t)width * cache->page_size > kMaxTokens) return BSP_EUNSUPPORTED;
    if (n == 0) return BSP_OK;
    return status(launch_extend({seqs, width, cache->pages, table, lens, refs, n, (int32_t *)scratch},
                                planes_args(cache, planes, plane_stride, data), rows, counts, pos, S(stream)));
}

bsp_status bsp_cache_release(int32_t seqs, int32_t width, int32_t pages, int32_t *table, int32_t *lens, int32_t *refs,
                             int32_t n, const int32_t *rows, void *stream) {
    if (const bsp_status st = check_pages(table, lens, refs, seqs, width, pages, n); st != BSP_OK) return st;
    if (n > 0 && !rows) return BSP_EINVAL;
    if (n == 0 || seqs == 0) return BSP_OK;
    return status(launch_release({seqs, width, pages, table, lens, refs, n, nullptr}, rows, S(stream)));
}

bsp_status bsp_cache_compact(const bsp_cache *cache, int32_t planes, int64_t plane_stride, void *data, int32_t seqs,
                             int32_t width, int32_t *table, int32_t *refs, int32_t *info, void *scratch, void *stream) {
    if (const bsp_status st = check_planes(cache, planes, plane_stride, data); st != BSP_OK) return st;
    if (seqs < 0 || width < 0 || (!table && (int64_t)seqs * width > 0) || !refs || !info || !scratch) return BSP_EINVAL;
    if (!aligned(scratch, 16)) return BSP_EINVAL;
    return status(launch_compact({seqs, width, cache->pages, table, nullptr, refs, 0, (int32_t *)scratch},
                                 planes_args(cache, planes, plane_stride, data), info, S(stream)));
}

bsp_status bsp_cache_copy(const bsp_cache *cache, int32_t planes, int64_t plane_stride, void *data, int32_t n,
                          const int32_t *src, const int32_t *dst, void *stream) {
    if (const bsp_status st = check_planes(cache, planes, plane_stride, data); st != BSP_OK) return st;
    if (n < 0 || (n > 0 && (!src || !dst))) return BSP_EINVAL;
    if (n == 0 || planes == 0) return BSP_OK;
    return status(launch_page_copy(planes_args(cache, planes, plane_stride, data), n, src, dst, S(stream)));
}

}  // extern "C"
