// k_q4: y = W x for W in 4 bits with group scales, on matrix instructions.
//
// Weights go from memory to the operand registers: a lane reads 16 bytes (32 codes) of one row, four
// lanes 128 columns; two exchanges between the quads (permlane swaps) give every lane the 8 codes of
// its place in each of four 16x16x32 products.  A code n becomes the bf16 1 + n / 16, by placing its
// bits in the mantissa of 1.0: two instructions for two codes.  What this adds, the constant, is
// taken out again by the sum's start value -1.5 sum(x), which a product with a constant operand gives
// once per group for all rows: 1 + n / 16 - 1.5 = (n - 8) / 16.  All products are exact and sums fp32;
// the group's scale multiplies its sum in fp32.
//
// Activations pass through LDS, a wave's own part of it, so the main loop has no barrier:
//  * one vector: 128 elements a chunk, in the order of the codes' pairs; a lane reads 16 bytes.
//  * more: rows of 16 NT elements of the feature-major array, loaded 16 bytes at a time at whatever
//    alignment; transposing LDS reads give a lane 4 rows of one column.  Rows of 64 elements are
//    twisted (32-byte pieces exchanged by bits 2 and 3 of the row), or the 16 rows that one read
//    touches would lie in the same banks.
//  * fp32 activations are cut into three bf16 (8 bits each, 24 in all), whose products are added.
// The waves of a workgroup take 128-column chunks in turn and are joined at the end.
#pragma once
#include "bsp_decode.h"
#include "bsp_decode_dev.h"

namespace bsp {

struct Q4Args {
    Q4Shape s;
    const void *x;
    const uint8_t *codes;
    const uint16_t *scales;
    const float *bias;
    void *y;
    int batch, relu, out_bf16;
    int waves;
};

constexpr int kQ4Chunk = 128;     // columns of a chunk
constexpr int kQ4Waves = 8;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Columns of x staged at a time, bf16 parts of an element, and a wave's LDS bytes.
template <typename X> constexpr int q4_parts() { return sizeof(X) == 4 ? 3 : 1; }
template <typename X, int NT> constexpr int q4_stage() {
    return sizeof(X) == 4 ? kQ4Chunk / NT : NT == 4 ? 64 : kQ4Chunk;
}
template <typename X, int NT, int MT, bool ONE> constexpr int q4_wave_lds() {
    constexpr int stage = ONE ? 4 * kQ4Chunk * 2 * q4_parts<X>() : q4_stage<X, NT>() * 16 * NT * 2 * q4_parts<X>();
    constexpr int join = (ONE ? 1 : 16 * NT) * (16 * MT + 4) * 4;
    return stage > join ? stage : join;
}

// 4 x 4 transpose over quads of lanes and registers.
__device__ __forceinline__ void q4_transpose(uint32_t *d) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto p = __builtin_amdgcn_permlane32_swap(d[i], d[i + 2], false, false);
        d[i] = p[0], d[i + 2] = p[1];
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const auto p = __builtin_amdgcn_permlane16_swap(d[i], d[i + 1], false, false);
        d[i] = p[0], d[i + 1] = p[1];
    }
}

// Eight codes as 1 + n / 16, in the order of pairs (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ bf16x8 q4_expand(uint32_t d) {
    const uint32_t mask = 0x00780078u, one = 0x3f803f80u;
    return as_bf16x8((u32x4){((d << 3) & mask) | one, ((d >> 1) & mask) | one, ((d >> 5) & mask) | one,
                                ((d >> 9) & mask) | one});
}

// The three bf16 whose sum an fp32 is (cut, not rounded, so that nothing overflows); Inf and NaN are
// their first part alone.
__device__ __forceinline__ void q4_cut(float x, uint16_t *p) {
    const uint32_t u = __float_as_uint(x);
    const bool finite = (u & 0x7f800000u) != 0x7f800000u;
    const float rest = x - __uint_as_float(u & 0xffff0000u);
    const uint32_t v = __float_as_uint(rest);
    const float last = rest - __uint_as_float(v & 0xffff0000u);
    p[0] = (uint16_t)((u >> 16) | ((!finite && (u & 0x007fffffu)) ? 0x40u : 0u));
    p[1] = finite ? (uint16_t)(v >> 16) : (uint16_t)0;
    p[2] = finite ? (uint16_t)(__float_as_uint(last) >> 16) : (uint16_t)0;
}
__device__ __forceinline__ void q4_cut(uint16_t x, uint16_t *p) { p[0] = x; }

// A workgroup: 16 MT rows, 16 NT vectors (ONE: one vector).
template <typename X, int G, int NT, int MT, bool ONE>
__global__ __launch_bounds__(64 * kQ4Waves, 2) void k_q4(Q4Args a) {
    constexpr int PARTS = q4_parts<X>(), GPC = kQ4Chunk / G, SPG = G / 32;   // groups of a chunk, steps of a group
    constexpr int STAGE = ONE ? kQ4Chunk : q4_stage<X, NT>();
    constexpr int PF = ONE ? 4 : 1;                                           // chunks in flight ahead
    constexpr int VE = 16 / sizeof(X);                                        // elements of a 16-byte load
    constexpr int NV = ONE ? 1 : STAGE * 16 * NT / VE / 64;                   // such loads of a lane and stage
    constexpr int WLDS = q4_wave_lds<X, NT, MT, ONE>();
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, quad = lane / 16;
    const int rows = a.s.rows, cols = a.s.cols, B = a.batch, W = a.waves;
    const int64_t row0 = (int64_t)blockIdx.x * (16 * MT);
    unsigned char *mine = lds + wave * WLDS;
    const X *x = (const X *)a.x;

    const int c0 = ONE ? 0 : blockIdx.y * (16 * NT), nc = ONE ? 1 : min(16 * NT, B - c0);   // its vectors

    const uint8_t *wp[MT];
    const uint16_t *sp = a.scales + row0 + quad * 4;
#pragma unroll
    for (int m = 0; m < MT; ++m) wp[m] = a.codes + min(row0 + 16 * m + r, (int64_t)rows - 1) * a.s.stride + quad * 16;
    const int n_chunks = (cols + kQ4Chunk - 1) / kQ4Chunk;

    struct Weights {
        u32x4 w[MT];
        u32x2 s[MT][GPC];
    };
    auto load_w = [&](int c, Weights &w) {   // past a row's end: its last 16 bytes, whose x is 0
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int64_t at = min((int64_t)c * 64, a.s.stride - 16 - quad * 16);
            w.w[m] = *(const u32x4 *)(wp[m] + at);
#pragma unroll
            for (int g = 0; g < GPC; ++g) {
                const int64_t group = min(c * GPC + g, a.s.n_groups - 1);
                w.s[m][g] = *(const u32x2 *)(sp + group * a.s.rows16 + min((int64_t)16 * m, a.s.rows16 - 16 - row0));
            }
        }
    };
    // one vector: elements 2 lane and 2 lane + 1 of a chunk, those past `cols` 0, each cut into its
    // parts, to their places: element k of 8 goes to place 2 (k % 4) + k / 4
    struct Pair {
        X e[2];
    };
    auto load_pair = [&](int64_t k0) {
        Pair p;
#pragma unroll
        for (int i = 0; i < 2; ++i) p.e[i] = k0 + 2 * lane + i < cols ? x[k0 + 2 * lane + i] : (X)0;
        return p;
    };
    auto store_pair = [&](const Pair &v, int slot) {
        uint16_t *at = (uint16_t *)mine + slot * kQ4Chunk * PARTS + (lane / 4) * 8 + (lane % 4 / 2) + (lane % 2) * 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint16_t p[3];
            q4_cut(v.e[i], p);
#pragma unroll
            for (int t = 0; t < PARTS; ++t) at[t * kQ4Chunk + 2 * i] = p[t];
        }
    };
    // more: rows of a stage, 16 bytes at a time.  What a row's last load takes past the vectors goes to
    // columns that no output has.
    constexpr int RS = 16 * NT, PLANE = STAGE * RS;
    struct Stage {
        u32x4 raw[NV];
    };
    auto twist = [](int row) { return NT == 4 ? (row >> 2 & 3) << 4 : 0; };   // in elements
    const int total = cols * B;
    auto whole = [&](int64_t k0) {   // a stage whose loads end within x
        return k0 + STAGE <= cols && (k0 + STAGE - 1) * B + c0 + (nc + VE - 1) / VE * VE <= total;
    };
    auto load_stage = [&](int64_t k0, Stage &v) {
        const X *p = x + k0 * B + c0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * 64 + lane) * VE, k = at / RS, c = at % RS;
            __builtin_memcpy(&v.raw[i], p + (c < nc ? k * B + c : 0), 16);
        }
    };
    // the last stages: rows past the last column of W are 0, and a load that would end past x begins
    // earlier (x has at least VE elements) and is shifted
    auto load_last = [&](int64_t k0, Stage &v) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * 64 + lane) * VE, k = at / RS, c = at % RS;
            const bool in = k0 + k < cols && c < nc;
            const int off = in ? (int)(k0 + k) * B + c0 + c : 0, from = min(off, total - VE);
            unsigned __int128 w;
            __builtin_memcpy(&w, x + from, 16);
            w = in ? w >> (8 * (int)sizeof(X) * (off - from)) : 0;
            __builtin_memcpy(&v.raw[i], &w, 16);
        }
    };
    auto store_stage = [&](const Stage &v) {
        uint16_t *base = (uint16_t *)mine;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = ((i * 64 + lane) * VE) ^ twist((i * 64 + lane) * VE / RS);
            if constexpr (PARTS == 1) {
                *(u32x4 *)(base + at) = v.raw[i];
            } else {
                uint16_t q[4][3];
#pragma unroll
                for (int j = 0; j < 4; ++j) q4_cut(__uint_as_float(v.raw[i][j]), q[j]);
#pragma unroll
                for (int t = 0; t < 3; ++t)
                    *(u32x2 *)(base + t * PLANE + at) = (u32x2){q[0][t] | (uint32_t)q[1][t] << 16, q[2][t] | (uint32_t)q[3][t] << 16};
            }
        }
    };
    auto stage_tiny = [&](int64_t k0) {   // of an x of fewer than VE elements
        uint16_t *base = (uint16_t *)mine;
        for (int e = lane; e < PLANE; e += 64) {
            const int k = e / RS, c = e % RS;
            uint16_t q[3];
            q4_cut(k0 + k < cols && c < nc ? x[(k0 + k) * B + c] : (X)0, q);
#pragma unroll
            for (int t = 0; t < PARTS; ++t) base[t * PLANE + (e ^ twist(k))] = q[t];
        }
    };
    int col_at[NT];                   // of the lane's transposing reads
#pragma unroll
    for (int t = 0; t < NT; ++t) col_at[t] = (t * 16 + r % 4 * 4) ^ twist(quad * 8 + r / 4 % 2 * 4);
    // the x operand of the step that begins at column k of the stage
    auto operand = [&](int k, int t, int part, int slot) {
        if constexpr (ONE) {
            return as_bf16x8(*(const u32x4 *)(mine + ((slot * PARTS + part) * kQ4Chunk + k + quad * 8) * 2));
        } else {
            const int row = k + quad * 8 + r / 4 % 2 * 4 + r / 8;
            unsigned char *p = mine + (part * PLANE + row * RS + col_at[t]) * 2;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(p));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(p + 4 * RS));
            const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
            return as_bf16x8((u32x4){l.x, l.y, h.x, h.y});
        }
    };

    f32x4 acc[MT][NT], sum[MT][NT], start[NT];
    const bf16x8 minus = as_bf16x8((u32x4){0xbfc0bfc0u, 0xbfc0bfc0u, 0xbfc0bfc0u, 0xbfc0bfc0u});   // -1.5
    const f32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[m][t] = zero;

    // the steps of columns [k, k + STAGE) of a chunk, whose codes are transposed in d
    auto multiply = [&](const uint32_t (*d)[4], const Weights &w, int k, int slot) {
#pragma unroll
        for (int s = 0; s < STAGE / 32; ++s) {
            const int step = k / 32 + s;                  // of the chunk
            const bool first = step % SPG == 0;
            bf16x8 wo[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) wo[m] = q4_expand(d[m][step]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (first) start[t] = zero;
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const bf16x8 xo = operand(s * 32, t, p, slot);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        sum[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wo[m], xo, first && p == 0 ? zero : sum[m][t], 0, 0, 0);
                    start[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(minus, xo, start[t], 0, 0, 0);
                }
            }
            if (step % SPG == SPG - 1)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const u32x2 sc = w.s[m][step / SPG];
                    const f32x4 f = {bf16_to_f32(sc.x & 0xffffu), __uint_as_float(sc.x & 0xffff0000u),
                                     bf16_to_f32(sc.y & 0xffffu), __uint_as_float(sc.y & 0xffff0000u)};
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[m][t] += f * (sum[m][t] + start[t]);
                }
        }
    };
    auto transpose = [&](const Weights &w, uint32_t (*d)[4]) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            d[m][0] = w.w[m].x, d[m][1] = w.w[m].y, d[m][2] = w.w[m].z, d[m][3] = w.w[m].w;
            q4_transpose(d[m]);
        }
    };
    auto fence = [&]() {   // a wave's LDS operations stay in order; the compiler's too
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    if constexpr (ONE) {
        Weights w[PF];
        Pair v[PF];
        for (int c = wave; c < n_chunks; c += PF * W) {
#pragma unroll
            for (int i = 0; i < PF; ++i) {
                load_w(c + i * W, w[i]);
                v[i] = load_pair((int64_t)(c + i * W) * kQ4Chunk);
            }
            fence();
#pragma unroll
            for (int i = 0; i < PF; ++i) store_pair(v[i], i);
            fence();
#pragma unroll
            for (int i = 0; i < PF; ++i) {
                uint32_t d[MT][4];
                transpose(w[i], d);
                multiply(d, w[i], 0, i);
            }
        }
    } else {
        Weights w;
        Stage v;
        auto load_x = [&](int64_t k0) {
            if (whole(k0))
                load_stage(k0, v);
            else if (k0 < (int64_t)n_chunks * kQ4Chunk && total >= VE)
                load_last(k0, v);
        };
        if (wave < n_chunks) load_w(wave, w);
        load_x((int64_t)wave * kQ4Chunk);
        for (int c = wave; c < n_chunks; c += W) {
            uint32_t d[MT][4];
            const Weights now = w;
            transpose(now, d);
            load_w(min(c + W, n_chunks - 1), w);
#pragma unroll
            for (int k = 0; k < kQ4Chunk; k += STAGE) {
                fence();
                if (total >= VE)
                    store_stage(v);
                else
                    stage_tiny((int64_t)c * kQ4Chunk + k);
                fence();
                load_x(k + STAGE < kQ4Chunk ? (int64_t)c * kQ4Chunk + k + STAGE : (int64_t)(c + W) * kQ4Chunk);
                multiply(d, now, k, 0);
            }
        }
    }

    // join the waves: [vector][row] of each in LDS
    constexpr int RW = 16 * MT + 4;
    float *o = (float *)mine;
    fence();
#pragma unroll
    for (int t = 0; t < NT; ++t)
        if (t * 16 + r < nc)
#pragma unroll
            for (int m = 0; m < MT; ++m) *(f32x4 *)(o + (t * 16 + r) * RW + m * 16 + quad * 4) = acc[m][t];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * MT * (ONE ? 1 : 16 * NT); i += 64 * W) {
        const int col = ONE ? 0 : i % (16 * NT), row = ONE ? i : i / (16 * NT);
        if (col >= nc || row0 + row >= rows) continue;
        float v = 0.f;
        for (int k = 0; k < W; ++k) v += ((const float *)(lds + k * WLDS))[col * RW + row];
        v = v * 16.f + (a.bias ? a.bias[row0 + row] : 0.f);
        if (a.relu && v < 0.f) v = 0.f;
        const int64_t at = (row0 + row) * B + c0 + col;
        if (a.out_bf16)
            ((uint16_t *)a.y)[at] = f32_to_bf16(v);
        else
            ((float *)a.y)[at] = v;
    }
}

template <typename X, int G, int NT, int MT, bool ONE>
hipError_t q4_run(const Q4Args &a, hipStream_t st) {
    constexpr int wave = q4_wave_lds<X, NT, MT, ONE>();
    if (kQ4Waves * wave > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)k_q4<X, G, NT, MT, ONE>,
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, kQ4Waves * wave);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)div_up64(a.s.rows, 16 * MT), ONE ? 1 : (unsigned)((a.batch + 16 * NT - 1) / (16 * NT)));
    k_q4<X, G, NT, MT, ONE><<<grid, 64 * a.waves, a.waves * wave, st>>>(a);
    return hipGetLastError();
}

template <typename X, int G>
hipError_t q4_pick(Q4Args a, hipStream_t st) {
    a.waves = std::min(kQ4Waves, (a.s.cols + kQ4Chunk - 1) / kQ4Chunk);
    if (a.batch == 1) return q4_run<X, G, 1, 1, true>(a, st);
    if (a.batch <= 16) return q4_run<X, G, 1, 1, false>(a, st);
    if (a.batch <= 32) return a.s.rows >= 32 * 256 ? q4_run<X, G, 2, 2, false>(a, st) : q4_run<X, G, 2, 1, false>(a, st);
    if (a.s.rows >= 32 * 192) return q4_run<X, G, 4, 2, false>(a, st);
    return q4_run<X, G, 4, 1, false>(a, st);
}

template <typename X>
hipError_t q4_linear(const Q4Args &a, hipStream_t st) {
    return a.s.group == 32 ? q4_pick<X, 32>(a, st) : a.s.group == 64 ? q4_pick<X, 64>(a, st) : q4_pick<X, 128>(a, st);
}

hipError_t q4_linear_bf16(const Q4Args &a, hipStream_t st);
hipError_t q4_linear_f32(const Q4Args &a, hipStream_t st);

}  // namespace bsp
