// FC layers with 4-bit weights and group scales: quantise, read back, and the forward for a few
// vectors.  Format (bsp.h): code n stands for scale * (n - 8); codes two to a byte in rows of
// `stride` bytes, scales bf16 [group][row].
#include <hip/hip_runtime.h>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"
#include "bsp_q4_mm.h"

namespace bsp {

namespace {

// Eight consecutive elements of a row, those at or past `n` read as 0.
template <typename E, bool VEC>
__device__ __forceinline__ void load8(const E *p, int n, float *v) {
    if (VEC && n >= 8) {
        alignas(16) E e[8];
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) ((uint4 *)e)[i] = ((const uint4 *)p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32<E>(e[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32<E>(p[i]) : 0.f;
}

// One workgroup: 16 rows x 128 columns, a thread 8 columns of a row.  The largest |w| of a group
// goes over its 4, 8 or 16 threads by lane exchanges, so w is read once and codes and scales are
// written once: bound by that traffic.
template <typename E, bool VEC>
__global__ __launch_bounds__(256) void k_q4_quantize(Q4Shape s, const E *__restrict__ w, const uint8_t *__restrict__ mask,
                                                     uint8_t *__restrict__ codes, uint16_t *__restrict__ scales) {
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    for (int64_t chunk = blockIdx.y; chunk * 64 < s.stride; chunk += gridDim.y) {
    const int64_t col = chunk * 128 + threadIdx.x % 16 * 8;
    const int n = row < s.rows ? (int)min((int64_t)8, s.cols - col) : 0;
    float v[8];
    load8<E, VEC>(w + row * s.cols + col, n, v);
    if (mask && n > 0) {
        const uint8_t *m = mask + row * s.cols + col;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n && !m[i]) v[i] = 0.f;
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
    for (int d = 1; d < s.group / 8; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const uint16_t sb = f32_to_bf16(top * (1.f / 7.f));
    const float sf = bf16_to_f32(sb);
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = sf == 0.f ? 0.f : fminf(fmaxf(rintf(v[i] / sf), -7.f), 7.f);
        if (i < n) packed |= (uint32_t)((int)q + 8) << (4 * i);
    }
    if (row < s.rows && col / 2 < s.stride) *(uint32_t *)(codes + row * s.stride + col / 2) = packed;
    if (row < s.rows16 && col % s.group == 0 && col < s.cols) scales[col / s.group * s.rows16 + row] = row < s.rows ? sb : 0;
    }
}

template <typename E, bool VEC>
__global__ __launch_bounds__(256) void k_q4_dequantize(Q4Shape s, const uint8_t *__restrict__ codes,
                                                       const uint16_t *__restrict__ scales, E *__restrict__ w) {
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    if (row >= s.rows) return;
    for (int64_t col = blockIdx.y * 128ll + threadIdx.x % 16 * 8; col < s.cols; col += gridDim.y * 128ll) {
    const uint32_t packed = *(const uint32_t *)(codes + row * s.stride + col / 2);
    const float sf = bf16_to_f32(scales[col / s.group * s.rows16 + row]);
    alignas(16) E e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = from_f32<E>((float)((int)(packed >> (4 * i) & 15) - 8) * sf);
    E *p = w + row * s.cols + col;
    const int n = (int)min((int64_t)8, s.cols - col);
    if (VEC && n == 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(e) / 16; ++i) ((uint4 *)p)[i] = ((uint4 *)e)[i];
        continue;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = e[i];
    }
}

// Rows that begin at multiples of 16 bytes are read and written in vectors.
template <typename E> bool in_vectors(const Q4Shape &s, const void *w) {
    return s.cols % (16 / (int)sizeof(E)) == 0 && (uintptr_t)w % 16 == 0;
}

template <typename E>
void quantize(const Q4Shape &s, const void *w, const uint8_t *mask, uint8_t *codes, uint16_t *scales, hipStream_t st) {
    const dim3 grid((unsigned)(s.rows16 / 16), (unsigned)std::min<int64_t>(div_up64(s.stride, 64), 65535));
    if (in_vectors<E>(s, w))
        k_q4_quantize<E, true><<<grid, 256, 0, st>>>(s, (const E *)w, mask, codes, scales);
    else
        k_q4_quantize<E, false><<<grid, 256, 0, st>>>(s, (const E *)w, mask, codes, scales);
}

template <typename E>
void dequantize(const Q4Shape &s, const uint8_t *codes, const uint16_t *scales, void *w, hipStream_t st) {
    const dim3 grid((unsigned)(s.rows16 / 16), (unsigned)std::min<int64_t>(div_up64(s.stride, 64), 65535));
    if (in_vectors<E>(s, w))
        k_q4_dequantize<E, true><<<grid, 256, 0, st>>>(s, codes, scales, (E *)w);
    else
        k_q4_dequantize<E, false><<<grid, 256, 0, st>>>(s, codes, scales, (E *)w);
}

}  // namespace

hipError_t launch_q4_quantize(const Q4Shape &s, int wdt, const void *w, const uint8_t *mask, uint8_t *codes,
                              uint16_t *scales, hipStream_t st) {
    if (wdt == BSP_F32)
        quantize<float>(s, w, mask, codes, scales, st);
    else
        quantize<uint16_t>(s, w, mask, codes, scales, st);
    return hipGetLastError();
}

hipError_t launch_q4_dequantize(const Q4Shape &s, int wdt, const uint8_t *codes, const uint16_t *scales, void *w,
                                hipStream_t st) {
    if (wdt == BSP_F32)
        dequantize<float>(s, codes, scales, w, st);
    else
        dequantize<uint16_t>(s, codes, scales, w, st);
    return hipGetLastError();
}

hipError_t launch_q4_linear(const Q4Shape &s, int batch, int in_dt, int out_dt, const void *x, const uint8_t *codes,
                            const uint16_t *scales, const float *bias, int relu, void *y, hipStream_t st) {
    const Q4Args a = {s, x, codes, scales, bias, y, batch, relu, out_dt == BSP_BF16, 0};
    return in_dt == BSP_F32 ? q4_linear_f32(a, st) : q4_linear_bf16(a, st);
}

}  // namespace bsp
