// What the attention kernels share: the steps of a wave, in registers only.
#pragma once
#include <hip/hip_runtime.h>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"
#include "bsp_paged.h"

namespace bsp {

namespace {

constexpr int kWaves = 4, kTile = 1024;   // waves of a workgroup; tokens whose places it keeps in LDS
constexpr int kBlock = 32;                // tokens by which work is cut up
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ int row_of(const AttnArgs &a, int b) { return a.rows ? a.rows[b] : b; }
__device__ __forceinline__ int len_of(const AttnArgs &a, int row) {
    const int len = (unsigned)row < (unsigned)a.seqs ? a.lens[row] : 0;
    return max(0, (int)min((int64_t)len, (int64_t)a.width * a.c.page_size));
}

// ONCE: past the caches.
template <bool ONCE, typename T> __device__ __forceinline__ T fetch(const T *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

// A kernel's (first) argument once more, for what is hardly ever reached: the compiler otherwise reads arguments that only
// this needs before all else, and those that all need later (64 sequences of 64 heads 49.5 us instead of 48.2).
template <typename T> __device__ __forceinline__ const T &argument_again() {
    const T *p = (const T *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *p;
}

// An output that is NaN where its probabilities are none has met an Inf: that times the second part of a bf16
// probability, which may be 0 or negative, or times one that fp32 holds as 0, is not what the probability itself gives.
// Which it is is told by the kinds of the values: the Inf that is among them, or NaN where both are, or a NaN.
// For the last step of an output alone, since the sums of parts would be NaN again: the others cost nothing (no more than 0.2
// us of 20), and calls that meet an Inf take long (1 sequence of 131072 tokens 2.6 ms, 64 over 32768 shared ones 12).
__device__ __forceinline__ bool any_nan(f32x4 v) { return v[0] != v[0] || v[1] != v[1] || v[2] != v[2] || v[3] != v[3]; }
constexpr int kNan = 1, kInf = 2, kMinusInf = 4;
__device__ __forceinline__ float told_by(int kinds) { return kinds == kInf ? INFINITY : kinds == kMinusInf ? -INFINITY : NAN; }
// The kinds of N values side by side at place(g), place(g + step), .. of n: add(e, kinds) takes those of value e and
// returns what is known of it, until all hold a NaN.  Bound by the latency of entry and value, AHEAD tokens at a time.
template <int N, int AHEAD, typename E, typename P, typename F>
__device__ __forceinline__ void kinds_of(const E *values, int n, int g, int step, P place, F add) {
    typedef E Some __attribute__((ext_vector_type(N)));
    for (int64_t i = g; i < n; i += AHEAD * step) {
        int64_t at[AHEAD];
        Some v[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) at[k] = place((int)min(i + k * step, (int64_t)n - 1));
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) v[k] = *(const Some *)(values + max(at[k], (int64_t)0));
        int all = kNan;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            int found = 0;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const E one = v[k][e];
                const float x = to_f32(one);
                if (at[k] >= 0) found |= x != x ? kNan : x == INFINITY ? kInf : x == -INFINITY ? kMinusInf : 0;
            }
            all &= add(e, found);
        }
        if (all) return;
    }
}

// What a wave loads and multiplies in one step, for head_dim up to DP: tokens of one key head, with N times 16
// query heads.
template <typename E, int DP> struct Step;

template <int DP> struct Step<uint16_t, DP> {
    static constexpr int TOK = 32, NK = DP / 32, VW = DP == 64 ? 4 : 8, NV = DP / (16 * VW);
    typedef uint32_t VRaw __attribute__((ext_vector_type(VW / 2)));
    typedef u32x4 Quad;            // a lane's part of a query's 32 dimensions
    u32x4 k[2][NK];
    VRaw v[8][NV];

    static __device__ __forceinline__ void load_q(u32x4 *q, const uint16_t *row, int quad) {
#pragma unroll
        for (int c = 0; c < NK; ++c) q[c] = *(const u32x4 *)(row + c * 32 + quad * 8);
    }
    // places of tokens r and 16 + r
    template <bool FULL, bool ONCE> __device__ __forceinline__ void load_k(const uint16_t *keys, const int64_t *ko, int quad, int D) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                if (!FULL && DP < 256 && c * 32 >= D) break;
                const int d = c * 32 + quad * 8;
                const bool in = FULL || d < D;
                k[t][c] = fetch<ONCE>((const u32x4 *)(keys + max(ko[t], (int64_t)0) + (in ? d : 0)));
                if (!in) k[t][c] = (u32x4){0, 0, 0, 0};
            }
    }
    // places of tokens 4 quad + i and 16 + 4 quad + i
    template <bool FULL, bool ONCE> __device__ __forceinline__ void load_v(const uint16_t *values, const int64_t *vo, int r, int D) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int h = 0; h < NV; ++h) {
                const int d = h * 16 * VW + r * VW;
                v[i][h] = fetch<ONCE>((const VRaw *)(values + max(vo[i], (int64_t)0) + (FULL || d < D ? d : 0)));
            }
    }
    __device__ __forceinline__ void clear_v(uint32_t dead) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (dead >> i & 1)
#pragma unroll
                for (int h = 0; h < NV; ++h) v[i][h] = (VRaw)0;
    }
    template <bool FULL> __device__ __forceinline__ void scores(const Quad *q, float *s, int D) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 c4 = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                if (!FULL && DP < 256 && c * 32 >= D) break;
                c4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k[t][c]), as_bf16x8(q[c]), c4, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * t + i] = c4[i];
        }
    }
    // A probability is the sum of two bf16, of which it keeps 16 bits (to 2^-16 of it): the second product
    // costs nothing that shows beneath the reads, and one rounded to a single bf16 would add as much
    // error as the output's own rounding.
    template <int N> __device__ __forceinline__ void outputs(const float (*p)[8], f32x4 (*acc)[NV][VW]) const {
        u32x4 b[N][2];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b[n][0][i] = pack_bf16(p[n][2 * i], p[n][2 * i + 1]);
                b[n][1][i] = pack_bf16(p[n][2 * i] - bf16_to_f32(b[n][0][i]), p[n][2 * i + 1] - __uint_as_float(b[n][0][i] & 0xffff0000u));
            }
#pragma unroll
        for (int h = 0; h < NV; ++h)
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                const uint32_t sel = j % 2 ? 0x07060302u : 0x05040100u;
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(v[2 * i + 1][h][j / 2], v[2 * i][h][j / 2], sel);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        acc[n][h][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(b[n][i]), acc[n][h][j], 0, 0, 0);
            }
    }
};

template <int DP> struct Step<float, DP> {
    static constexpr int TOK = 16, NK = DP / 16, VW = 4, NV = DP / 64;
    typedef f32x4 Quad;            // a lane's part of a query's 16 dimensions
    f32x4 k[NK];
    f32x4 v[4][NV];

    static __device__ __forceinline__ void load_q(f32x4 *q, const float *row, int quad) {
#pragma unroll
        for (int c = 0; c < NK; ++c) q[c] = *(const f32x4 *)(row + c * 16 + quad * 4);
    }
    template <bool FULL, bool ONCE> __device__ __forceinline__ void load_k(const float *keys, const int64_t *ko, int quad, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            if (!FULL && DP < 256 && c * 16 >= D) break;
            const int d = c * 16 + quad * 4;
            const bool in = FULL || d < D;
            k[c] = fetch<ONCE>((const f32x4 *)(keys + max(ko[0], (int64_t)0) + (in ? d : 0)));
            if (!in) k[c] = (f32x4){0, 0, 0, 0};
        }
    }
    template <bool FULL, bool ONCE> __device__ __forceinline__ void load_v(const float *values, const int64_t *vo, int r, int D) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < NV; ++h) {
                const int d = h * 64 + r * 4;
                v[i][h] = fetch<ONCE>((const f32x4 *)(values + max(vo[i], (int64_t)0) + (FULL || d < D ? d : 0)));
            }
    }
    __device__ __forceinline__ void clear_v(uint32_t dead) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (dead >> i & 1)
#pragma unroll
                for (int h = 0; h < NV; ++h) v[i][h] = (f32x4){0, 0, 0, 0};
    }
    template <bool FULL> __device__ __forceinline__ void scores(const Quad *q, float *s, int D) const {
        f32x4 c4[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};   // two chains, or each product waits for the one before
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            if (!FULL && DP < 256 && c * 16 >= D) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) c4[i % 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][i], q[c][i], c4[i % 2], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = c4[0][i] + c4[1][i];
    }
    template <int N> __device__ __forceinline__ void outputs(const float (*p)[4], f32x4 (*acc)[NV][VW]) const {
#pragma unroll
        for (int h = 0; h < NV; ++h)
#pragma unroll
            for (int j = 0; j < VW; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        acc[n][h][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][h][j], p[n][i], acc[n][h][j], 0, 0, 0);
    }
};

}  // namespace

}  // namespace bsp
