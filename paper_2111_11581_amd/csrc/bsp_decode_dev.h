// Device helpers of the decode operators.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bsp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// A value that all lanes of the wave hold, in a scalar register.
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float bf16_to_f32(uint32_t h) { return __uint_as_float(h << 16); }
// To the nearest bf16, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t f32_to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return bf16_to_f32(v); }
template <typename E> __device__ __forceinline__ E from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_f32<uint16_t>(float v) { return f32_to_bf16(v); }

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Scans over the wave's 64 lanes, all of which are there; 0 adds nothing to `join`.  By moves within and between rows of
// 16 lanes; with shuffles, which go through LDS, the sampling of 64 rows of 131072 tokens takes 72.1 us instead of 64.4.
template <int CONTROL, int ROWS, typename T> __device__ __forceinline__ T moved(T v) {
    if constexpr (sizeof(T) == 8) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = moved<CONTROL, ROWS>((uint32_t)u), hi = moved<CONTROL, ROWS>((uint32_t)(u >> 32));
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    } else {
        return (T)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, ROWS, 0xf, false);
    }
}
template <typename T, typename F> __device__ __forceinline__ T wave_scan(T v, F join) {
    v = join(v, moved<0x111, 0xf>(v));   // from 1, 2, 4 and 8 lanes below, within a row
    v = join(v, moved<0x112, 0xf>(v));
    v = join(v, moved<0x114, 0xf>(v));
    v = join(v, moved<0x118, 0xf>(v));
    v = join(v, moved<0x142, 0xa>(v));   // the last lane of the row below, for rows 1 and 3
    v = join(v, moved<0x143, 0xc>(v));   // lane 31, for rows 2 and 3
    return v;
}
// Of one lane, for all.
template <typename T> __device__ __forceinline__ T of_lane(T v, int lane) {
    if constexpr (sizeof(T) == 8) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        return __builtin_bit_cast(T, (uint64_t)of_lane((uint32_t)(u >> 32), lane) << 32 | of_lane((uint32_t)u, lane));
    } else {
        return (T)__builtin_amdgcn_readlane((int)v, lane);
    }
}
template <typename T, typename F> __device__ __forceinline__ T wave_all(T v, F join) { return of_lane(wave_scan(v, join), 63); }
struct Sum {
    template <typename T> __device__ __forceinline__ T operator()(T x, T y) const { return x + y; }
};
struct Largest {
    template <typename T> __device__ __forceinline__ T operator()(T x, T y) const { return x > y ? x : y; }
};

}  // namespace bsp
