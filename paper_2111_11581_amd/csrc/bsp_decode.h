// Launch interface of the decode operators: 4-bit FC layers, attention over a paged cache, and
// the care of its pages.  Arguments are checked at the C entry points (bsp_api_decode.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include "bsp_common.h"

namespace bsp {

// ---- 4-bit weights ----
struct Q4Shape {
    int rows, cols, group;
    int n_groups, rows16;         // groups of a row; rows rounded up to 16 (row length of scales)
    int64_t stride;               // bytes from a row of codes to the next
};
inline Q4Shape q4_shape(int rows, int cols, int group) {
    Q4Shape s;
    s.rows = rows, s.cols = cols, s.group = group;
    s.n_groups = (int)(((int64_t)cols + group - 1) / group);
    s.rows16 = (int)(((int64_t)rows + 15) / 16 * 16);
    s.stride = (((int64_t)cols + 1) / 2 + 15) / 16 * 16;
    return s;
}
hipError_t launch_q4_quantize(const Q4Shape &s, int wdt, const void *w, const uint8_t *mask, uint8_t *codes,
                              uint16_t *scales, hipStream_t st);
hipError_t launch_q4_dequantize(const Q4Shape &s, int wdt, const uint8_t *codes, const uint16_t *scales, void *w,
                                hipStream_t st);
hipError_t launch_q4_linear(const Q4Shape &s, int batch, int in_dt, int out_dt, const void *x, const uint8_t *codes,
                            const uint16_t *scales, const float *bias, int relu, void *y, hipStream_t st);

// ---- paged cache ----
struct CacheArgs {
    int dtype, order, pages, page_size, kv_heads, head_dim;
    int64_t page_stride, head_stride, slot_stride;   // elements
    FastDiv div_page;             // token -> page of the sequence
};
inline CacheArgs cache_args(const bsp_cache &c) {
    CacheArgs a;
    a.dtype = c.dtype, a.order = c.order, a.pages = c.pages, a.page_size = c.page_size;
    a.kv_heads = c.kv_heads, a.head_dim = c.head_dim;
    const int64_t page = (int64_t)c.page_size * c.kv_heads * c.head_dim;
    a.page_stride = c.page_stride ? c.page_stride : page;
    a.head_stride = c.order == BSP_HEAD_MAJOR ? (int64_t)c.page_size * c.head_dim : c.head_dim;
    a.slot_stride = c.order == BSP_HEAD_MAJOR ? c.head_dim : (int64_t)c.kv_heads * c.head_dim;
    a.div_page = make_fastdiv((unsigned)c.page_size);
    return a;
}

// Whether keys and values of a layer span more than half of the last-level cache.
constexpr int64_t kLarge = 128 << 20;   // bytes
inline bool past_caches(const CacheArgs &c) {
    return c.page_stride * c.pages > kLarge / (c.dtype == BSP_F32 ? 8 : 4);
}

struct AppendArgs {
    CacheArgs c;
    const void *k, *v;
    void *keys, *values;
    bsp_strides ks, vs;
    const int32_t *table, *rows, *pos;
    int n, seqs, width;
};
hipError_t launch_append(const AppendArgs &a, hipStream_t st);

struct AttnArgs {
    CacheArgs c;
    const void *q, *keys, *values;
    void *y;
    float *lse;
    bsp_strides qs, ys;
    const int32_t *table, *rows, *lens;
    int batch, heads, group, seqs, width, window;
    float scale;
    void *workspace;
    int shares;                   // set by launch_attention: workgroups that the work is cut for, 0: one a unit
    int head_groups;              // set by launch_attention: of up to 16 query heads of a key head
};
int64_t attention_workspace(const CacheArgs &c, int batch, int heads, int width);
hipError_t launch_attention(AttnArgs a, hipStream_t st);

// ---- pages ----
struct PagesArgs {
    int seqs, width, pages;
    int32_t *table, *lens, *refs;
    int n;
    int32_t *scratch;
};
struct PlanesArgs {
    CacheArgs c;
    int planes;
    int64_t plane_stride;
    void *data;
};
int64_t pages_scratch(int pages, int width, int n);
hipError_t launch_fork(const PagesArgs &a, const int32_t *parents, const int32_t *children, hipStream_t st);
hipError_t launch_extend(const PagesArgs &a, const PlanesArgs &d, const int32_t *rows, const int32_t *counts,
                         int32_t *pos, hipStream_t st);
hipError_t launch_release(const PagesArgs &a, const int32_t *rows, hipStream_t st);
hipError_t launch_compact(const PagesArgs &a, const PlanesArgs &d, int32_t *info, hipStream_t st);
hipError_t launch_page_copy(const PlanesArgs &d, int n, const int32_t *src, const int32_t *dst, hipStream_t st);

}  // namespace bsp
