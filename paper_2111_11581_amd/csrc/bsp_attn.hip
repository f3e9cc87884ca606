// Attention of one new token over a paged cache, and the write of its key and value.
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_decode.h"

namespace bsp {

namespace {

__device__ __forceinline__ float bf16_to_f32(uint32_t h) { return __uint_as_float(h << 16); }
// Round to nearest even; NaN stays NaN.
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40u);
    return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}
__device__ __forceinline__ float ld(const float *p) { return *p; }
__device__ __forceinline__ float ld(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void st(float *p, float v) { *p = v; }
__device__ __forceinline__ void st(uint16_t *p, float v) { *p = f32_to_bf16(v); }

// Page of token t of a sequence, or -1 where the entry holds nothing.
__device__ __forceinline__ int page_of(const CacheArgs &c, const int32_t *row, uint32_t t, uint32_t *slot) {
    const uint32_t e = fdiv(t, c.div_page);
    *slot = t - e * (uint32_t)c.page_size;
    const int p = row[e];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
}

// A thread copies one element of a token's key or value.
template <typename E>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
    const int i = blockIdx.x, dims = a.c.kv_heads * a.c.head_dim;
    const int row = a.rows ? a.rows[i] : i, pos = a.pos[i];
    if ((unsigned)row >= (unsigned)a.seqs || pos < 0) return;
    if (pos >= (int64_t)a.width * a.c.page_size) return;
    uint32_t slot;
    const int page = page_of(a.c, a.table + (int64_t)row * a.width, (uint32_t)pos, &slot);
    if (page < 0) return;
    const E *src = (const E *)(blockIdx.y ? a.v : a.k);
    const bsp_strides s = blockIdx.y ? a.vs : a.ks;
    E *dst = (E *)(blockIdx.y ? a.values : a.keys) + page * a.c.page_stride + slot * a.c.slot_stride;
    for (int j = threadIdx.x; j < dims; j += blockDim.x) {
        const int h = j / a.c.head_dim, d = j - h * a.c.head_dim;
        dst[h * a.c.head_stride + d] = src[i * s.seq + h * s.head + d * s.dim];
    }
}

// One workgroup per query head and sequence: a wave takes every fourth token, a lane up to 4
// dimensions; the waves' running maxima, sums and outputs are joined at the end.
template <typename E>
__global__ __launch_bounds__(256) void k_attention(AttnArgs a) {
    __shared__ float sm[4], sl[4], so[4][256];
    const int h = blockIdx.x % a.heads, b = blockIdx.x / a.heads, wave = threadIdx.x / 64, lane = threadIdx.x % 64, D = a.c.head_dim;
    const int row = a.rows ? a.rows[b] : b;
    int len = (unsigned)row < (unsigned)a.seqs ? a.lens[row] : 0;
    len = (int)min((int64_t)len, (int64_t)a.width * a.c.page_size);
    const int first = a.window && len > a.window ? len - a.window : 0;
    const E *q = (const E *)a.q + b * a.qs.seq + h * a.qs.head;
    float qv[4], o[4] = {}, m = -INFINITY, l = 0.f;
    for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < D ? ld(q + (lane + 64 * i) * a.qs.dim) * a.scale : 0.f;
    for (int t = first + wave; t < len; t += 4) {
        uint32_t slot;
        const int page = page_of(a.c, a.table + (int64_t)row * a.width, (uint32_t)t, &slot);
        if (page < 0) continue;
        const int64_t at = page * a.c.page_stride + h / a.group * a.c.head_stride + slot * a.c.slot_stride;
        const E *k = (const E *)a.keys + at, *v = (const E *)a.values + at;
        float s = 0.f;
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < D) s += qv[i] * ld(k + lane + 64 * i);
        for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
        const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
        const float keep = expf(m - ref), p = expf(s - ref);
        l = l * keep + p;
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < D) o[i] = o[i] * keep + p * ld(v + lane + 64 * i);
        m = top;
    }
    if (lane == 0) sm[wave] = m, sl[wave] = l;
    for (int i = 0; i < 4; ++i) so[wave][lane + 64 * i] = o[i];
    __syncthreads();
    float top = -INFINITY, sum = 0.f, out = 0.f;
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < 4; ++w) {
        const float f = expf(sm[w] - ref);
        sum += sl[w] * f;
        out += so[w][threadIdx.x] * f;
    }
    if ((int)threadIdx.x < D) {
        E *y = (E *)a.y + b * a.ys.seq + h * a.ys.head + threadIdx.x * a.ys.dim;
        st(y, sum == 0.f ? 0.f : out / sum);
    }
    if (a.lse && threadIdx.x == 0) a.lse[(int64_t)b * a.heads + h] = ref + logf(sum);
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t st) {
    const dim3 grid(a.n, 2);
    if (a.c.dtype == BSP_F32)
        k_append<uint32_t><<<grid, 256, 0, st>>>(a);
    else
        k_append<uint16_t><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

int64_t attention_workspace(const CacheArgs &, int, int, int) { return 0; }

hipError_t launch_attention(const AttnArgs &a, hipStream_t st) {
    const dim3 grid(a.heads * a.batch);
    if (a.c.dtype == BSP_F32)
        k_attention<float><<<grid, 256, 0, st>>>(a);
    else
        k_attention<uint16_t><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace bsp
