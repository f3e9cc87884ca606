// FC layers with 4-bit weights and group scales: quantise, read back, launches.  Format (bsp.h): code
// n stands for scale * (n - 8); codes two to a byte in rows of `stride` bytes, scales bf16
// [group][row].
#include <hip/hip_runtime.h>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"
#include "bsp_q4_mm.h"

namespace bsp {

namespace {

// Both kernels: a workgroup takes 16 rows x 128 columns, a thread 8 columns of a row.  Places past the
// end are read at the row's own start (or the last row's) and dropped.  With 2 or 4 such tiles to a
// workgroup and all of their loads first, 4096 x 4096 fp32 there and back took 5 and 8 % longer.
struct Place {
    int64_t row, col;
    __device__ __forceinline__ Place(const Q4Shape &s) {
        const unsigned tiles = (unsigned)((s.stride + 63) / 64), down = blockIdx.x / tiles;
        row = (int64_t)down * 16 + threadIdx.x / 16;
        col = (int64_t)(blockIdx.x - down * tiles) * 128 + threadIdx.x % 16 * 8;
    }
};

// Eight elements of a row (of w, or of the mask) from column `col` on, as they are in memory.  VEC: rows
// of w begin at multiples of 16 bytes, so that a vector is inside or outside as a whole; what is
// outside is read at the row's start, and since nothing is read again, past the caches (4096 x 4096
// fp32 there and back 31 us, through them 33.5).  Else all eight at once at whatever alignment, and
// one by one only at a row's end (3000 x 4001 bf16 37 us one by one, 29.5 so; without VEC the first
// takes 40).
template <typename T, bool VEC, int BYTES> struct Eight {
    typedef uint32_t Raw __attribute__((ext_vector_type(BYTES / 4)));
    static constexpr int V = 8 * sizeof(T) / BYTES, N = 8 / V;   // vectors, elements of each
    Raw v[V];
    __device__ __forceinline__ void load(const T *row, int64_t col, int64_t cols) {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = __builtin_nontemporal_load((const Raw *)(row + (col + i * N < cols ? col + i * N : 0)));
        } else if (col + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < V; ++i) __builtin_memcpy(&v[i], row + col + i * N, BYTES);
        } else {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = row[col + i < cols ? col + i : 0];
            __builtin_memcpy(v, e, sizeof e);
        }
    }
    __device__ __forceinline__ void store(T *row, int64_t col, int64_t cols) const {
        if (VEC) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (col + i * N < cols) *(Raw *)(row + col + i * N) = v[i];
        } else if (col + 8 <= cols) {
#pragma unroll
            for (int i = 0; i < V; ++i) __builtin_memcpy(row + col + i * N, &v[i], BYTES);
        } else {
            T e[8];
            __builtin_memcpy(e, v, sizeof e);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < cols) row[col + i] = e[i];
        }
    }
    __device__ __forceinline__ uint32_t word(int i) const { return v[i / N][i % N * sizeof(T) / 4]; }
};
template <bool VEC> __device__ __forceinline__ float element(const Eight<float, VEC, 16> &e, int i) {
    return __uint_as_float(e.word(i));
}
template <bool VEC> __device__ __forceinline__ float element(const Eight<uint16_t, VEC, 16> &e, int i) {
    return bf16_to_f32((uint16_t)(e.word(i) >> (i % 2 * 16)));
}

// The largest |w| of a group goes over its 4, 8 or 16 threads by lane exchanges, so w is read once and
// codes and scales are written once: bound by that traffic (4096 x 4096 fp32: 76 MB in 16 us, 4.7 TB/s;
// 512 x 4608 bf16 with a mask 4.7 us).
template <typename E, bool VEC, bool MASK>
__global__ __launch_bounds__(256) void k_q4_quantize(Q4Shape s, const E *__restrict__ w, const uint8_t *__restrict__ mask,
                                                     uint8_t *__restrict__ codes, uint16_t *__restrict__ scales) {
    const Place at(s);
    const int64_t row = at.row, col = at.col, from = min(row, s.rows - 1ll) * s.cols;
    Eight<E, VEC, 16> x;
    x.load(w + from, col, s.cols);
    Eight<uint8_t, VEC, 4> m;   // with VEC, cols is a multiple of 4
    if constexpr (MASK) m.load(mask + from, col, s.cols);
    const int n = row < s.rows ? (int)min((int64_t)8, s.cols - col) : 0;
    float v[8], top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = i < n ? element(x, i) : 0.f;
        if constexpr (MASK) v[i] = m.word(i) >> (i % 4 * 8) & 255 ? v[i] : 0.f;
        top = fmaxf(top, fabsf(v[i]));
    }
    for (int d = 1; d < s.group / 8; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const uint16_t sb = f32_to_bf16(top * (1.f / 7.f));
    const float sf = bf16_to_f32(sb);
    float q[8];
    if (sf >= 0x1p-100f && sf <= 0x1p100f) {
        // v / sf to the last bit from the correctly rounded 1 / sf and one exact remainder (Markstein's
        // correction); an odd multiple of sf / 2 is exact, so ties are the division's.  20.4 -> 18.2 us
        const float r = 1.f / sf;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float near = v[i] * r;
            q[i] = __builtin_fmaf(__builtin_fmaf(-near, sf, v[i]), r, near);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = sf == 0.f ? 0.f : v[i] / sf;
    }
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)   // 1.5 * 2^23 + 8 rounds to the nearest code, which is left in the lowest bits
        packed |= (__float_as_uint(fminf(fmaxf(q[i], -7.f), 7.f) + 12582920.f) & 15) << (4 * i);
    if (n < 8) packed &= n > 0 ? (1u << (4 * n)) - 1 : 0;
    if (row < s.rows && col / 2 < s.stride) *(uint32_t *)(codes + row * s.stride + col / 2) = packed;
    if (row < s.rows16 && col % s.group == 0 && col < s.cols)
        scales[col / s.group * s.rows16 + row] = row < s.rows ? sb : 0;
}

// Bound by the same traffic the other way: 15.2 us, 5.0 TB/s; 512 x 4608 bf16 3.6 us.
template <typename E, bool VEC>
__global__ __launch_bounds__(256) void k_q4_dequantize(Q4Shape s, const uint8_t *__restrict__ codes,
                                                       const uint16_t *__restrict__ scales, E *__restrict__ w) {
    const Place at(s);
    if (at.row >= s.rows || at.col >= s.cols) return;
    const uint32_t packed = *(const uint32_t *)(codes + at.row * s.stride + at.col / 2);
    const float sf = bf16_to_f32(scales[at.col / s.group * s.rows16 + at.row]);
    E e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = from_f32<E>((float)((int)(packed >> (4 * i) & 15) - 8) * sf);
    Eight<E, VEC, 16> y;
    __builtin_memcpy(y.v, e, sizeof e);
    y.store(w + at.row * s.cols, at.col, s.cols);
}

// Rows that begin at multiples of 16 bytes (of the mask: 4) are read and written in vectors.
template <typename E> bool in_vectors(const Q4Shape &s, const void *w, const void *mask) {
    return s.cols % (16 / (int)sizeof(E)) == 0 && (uintptr_t)w % 16 == 0 && (uintptr_t)mask % 4 == 0;
}

dim3 prepare_grid(const Q4Shape &s) {
    return dim3((unsigned)(s.rows16 / 16 * div_up64(s.stride, 64)));
}

template <typename E, bool VEC>
void quantize(const Q4Shape &s, const E *w, const uint8_t *mask, uint8_t *codes, uint16_t *scales, hipStream_t st) {
    if (mask)
        k_q4_quantize<E, VEC, true><<<prepare_grid(s), 256, 0, st>>>(s, w, mask, codes, scales);
    else
        k_q4_quantize<E, VEC, false><<<prepare_grid(s), 256, 0, st>>>(s, w, mask, codes, scales);
}

template <typename E>
void quantize(const Q4Shape &s, const void *w, const uint8_t *mask, uint8_t *codes, uint16_t *scales, hipStream_t st) {
    if (in_vectors<E>(s, w, mask))
        quantize<E, true>(s, (const E *)w, mask, codes, scales, st);
    else
        quantize<E, false>(s, (const E *)w, mask, codes, scales, st);
}

template <typename E>
void dequantize(const Q4Shape &s, const uint8_t *codes, const uint16_t *scales, void *w, hipStream_t st) {
    if (in_vectors<E>(s, w, nullptr))
        k_q4_dequantize<E, true><<<prepare_grid(s), 256, 0, st>>>(s, codes, scales, (E *)w);
    else
        k_q4_dequantize<E, false><<<prepare_grid(s), 256, 0, st>>>(s, codes, scales, (E *)w);
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
