// y = W x for W in 4 bits with group scales, on matrix instructions: k_q4_one for one vector, k_q4 for
// more.
//
// Weights go from memory to the operand registers: a lane reads 16 bytes (32 codes) of one row, four
// lanes 128 columns; two exchanges between the quads (permlane swaps) give every lane the 8 codes of
// its place in each of four 16x16x32 products.  A code n becomes (n - 8) / 128 in bf16, exactly, so that
// a weight of 0 takes no part in a sum, however large its activation is.  All products are exact and
// sums fp32; the group's scale multiplies its sum in fp32.  fp32 activations are cut into three bf16
// (8 bits each, 24 in all), whose products are added.
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

template <typename X> constexpr int q4_parts() { return sizeof(X) == 4 ? 3 : 1; }   // bf16 parts of an element

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

// Eight codes as (n - 8) / 128, in the order of pairs (0, 2), (1, 3), (4, 6), (5, 7).  An fp8 (e4m3) whose
// lower half counts 0 .. 8 is that many 512ths, so sign and magnitude, worked out for all eight at once,
// are spread to a byte each and converted two at a time: 15 instructions.  (1 + n / 16 by placing n in
// the mantissa of 1.0 takes 8, but the 1.5 x to be taken off again leaves its own rounding error of every
// x, of a removed weight's too: 1e-4 of an output where three such x are 10^4 times the rest.  One vector
// 1 to 14 % faster so, 4096 x 4096 4.0 us for 4.5; 64 vectors the same.)
__device__ __forceinline__ bf16x8 q4_expand(uint32_t d) {
    const uint32_t minus = ~(d >> 3) & 0x11111111u;                  // n < 8
    const uint32_t size = (d ^ (0x88888888u - minus)) + minus;       // n ^ 8, or (n ^ 7) + 1
    const uint32_t even = (size & 0x0f0f0f0fu) | (minus << 7 & 0xf0f0f0f0u);
    const uint32_t odd = (size >> 4 & 0x0f0f0f0fu) | (minus << 3 & 0xf0f0f0f0u);
    auto pair = [](bf16x2 v) { return __builtin_bit_cast(uint32_t, v); };
    return as_bf16x8((u32x4){pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 4.f, false)),
                             pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 4.f, false)),
                             pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 4.f, true)),
                             pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 4.f, true))});
}

// The upper halves of a pair, and what they leave of each.
__device__ __forceinline__ uint32_t q4_upper(float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float q4_rest(float a) { return a - __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
// Pairs of elements as pairs of each of their bf16 parts.  An fp32 is the sum of three bf16, cut, not
// rounded, so that nothing overflows; of an Inf or NaN the second is NaN.
__device__ __forceinline__ void q4_cut(float a, float b, uint32_t *p) {
    p[0] = q4_upper(a, b);
    a = q4_rest(a), b = q4_rest(b);
    p[1] = q4_upper(a, b);
    p[2] = q4_upper(q4_rest(a), q4_rest(b));
}
__device__ __forceinline__ void q4_cut(uint16_t a, uint16_t b, uint32_t *p) { p[0] = a | (uint32_t)b << 16; }

// Where a lane finds codes: 32-bit offsets from the workgroup's first row, so that an address is a
// scalar base and one register.  Past the last row the last one is read again.
template <int MT> struct Q4Lane {
    const uint8_t *codes;
    uint32_t at[MT], quad16, last;
    const uint16_t *scales[MT];
    __device__ __forceinline__ Q4Lane(const Q4Args &a, int64_t row0, int r, int quad)
        : codes(a.codes + row0 * a.s.stride), quad16(quad * 16), last((uint32_t)a.s.stride - 16) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            at[m] = (uint32_t)min((int64_t)16 * m + r, a.s.rows - 1 - row0) * (uint32_t)a.s.stride;
            scales[m] = a.scales + min(row0 + 16 * m, (int64_t)a.s.rows16 - 16);
        }
    }
};

// Codes and scales of a 128-column chunk of MT row tiles, as a lane holds them.
template <int G, int MT> struct Q4Weights {
    static constexpr int GPC = kQ4Chunk / G;   // groups of a chunk
    u32x4 w[MT];
    u32x2 s[MT][GPC];

    // Past a row's end its last 16 bytes are read again, whose x is 0; past the last group the last.
    __device__ __forceinline__ void load(const Q4Args &a, const Q4Lane<MT> &l, int chunk) {
        const uint32_t col = min((uint32_t)chunk * 64 + l.quad16, l.last);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            w[m] = *(const u32x4 *)(l.codes + (l.at[m] + col));
#pragma unroll
            for (int g = 0; g < GPC; ++g)
                s[m][g] = *(const u32x2 *)((const uint8_t *)(l.scales[m] + (int64_t)min(chunk * GPC + g, a.s.n_groups - 1) * a.s.rows16) +
                                           (l.quad16 >> 1));
        }
    }
    __device__ __forceinline__ void codes(int m, uint32_t *d) const {
        d[0] = w[m].x, d[1] = w[m].y, d[2] = w[m].z, d[3] = w[m].w;
        q4_transpose(d);
    }
    __device__ __forceinline__ f32x4 scale(int m, int g) const {
        return (f32x4){bf16_to_f32(s[m][g].x & 0xffffu), __uint_as_float(s[m][g].x & 0xffff0000u),
                       bf16_to_f32(s[m][g].y & 0xffffu), __uint_as_float(s[m][g].y & 0xffff0000u)};
    }
};

// The products of `steps` 32-column steps of one group, from step `first` of a chunk: x operands xo of
// NT vector tiles, codes d of the MT row tiles.
template <int G, int MT, int NT, int PARTS, int US>
__device__ __forceinline__ void q4_unit(const Q4Weights<G, MT> &w, const uint32_t (*d)[4], int first,
                                        const bf16x8 (*xo)[NT][PARTS], f32x4 (*acc)[NT]) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        f32x4 sum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < US; ++s) {
            const bf16x8 wo = q4_expand(d[m][first + s]);
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wo, xo[s][t][p], sum[t], 0, 0, 0);
        }
        const f32x4 f = w.scale(m, first / (G / 32));
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[m][t] += f * sum[t];
        if (MT > 1) __builtin_amdgcn_sched_barrier(0);   // or all tiles' sums are begun at once, and spill
    }
}

// Sum over the waves that share rows, bias, ReLU and the store of one output.
__device__ __forceinline__ void q4_store(const Q4Args &a, float v, int64_t row, int col) {
    v = v * 128.f + (a.bias ? a.bias[row] : 0.f);
    if (a.relu && v < 0.f) v = 0.f;
    const int64_t at = row * a.batch + col;
    if (a.out_bf16)
        ((uint16_t *)a.y)[at] = f32_to_bf16(v);
    else
        ((float *)a.y)[at] = v;
}

// One vector.  A workgroup computes 16 rows; its waves take chunks in turn, four at a time in flight,
// and are joined at the end.  A wave keeps x of its chunks in its own part of LDS, in the order of the
// codes' pairs, and a lane reads the 16 bytes of its 8 columns (all 16 columns of the operand are the
// vector).
template <typename X, int G>
__global__ __launch_bounds__(64 * kQ4Waves, 4) void k_q4_one(Q4Args a) {
    constexpr int PARTS = q4_parts<X>(), PF = 4, SPG = G / 32;
    __shared__ __attribute__((aligned(16))) uint16_t s_x[kQ4Waves][PF][PARTS][kQ4Chunk];
    __shared__ f32x4 s_o[kQ4Waves][4];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, quad = lane / 16;
    const int W = a.waves, cols = a.s.cols;
    const int64_t row0 = (int64_t)blockIdx.x * 16;
    const Q4Lane<1> at(a, row0, r, quad);
    const X *x = (const X *)a.x;
    const int n_chunks = (cols + kQ4Chunk - 1) / kQ4Chunk;
    f32x4 acc[1][1] = {{{0, 0, 0, 0}}};
    Q4Weights<G, 1> w[PF];
    X v[PF][2];
    for (int c = wave; c < n_chunks; c += PF * W) {
#pragma unroll
        for (int i = 0; i < PF; ++i) {
            const uint32_t k = (uint32_t)(c + i * W) * kQ4Chunk + lane;   // elements lane and lane + 64 of the chunk
            v[i][0] = x[min(k, (uint32_t)cols - 1)], v[i][1] = x[min(k + 64, (uint32_t)cols - 1)];
            w[i].load(a, at, min(c + i * W, n_chunks - 1));
        }
        // a wave's LDS operations stay in order; the fences hold the compiler to it
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < PF; ++i) {
            const int k = (c + i * W) * kQ4Chunk + lane;
            uint32_t p[3];
            q4_cut(k < cols ? v[i][0] : (X)0, k + 64 < cols ? v[i][1] : (X)0, p);
#pragma unroll
            for (int t = 0; t < PARTS; ++t) {   // elements 1 and 2, 5 and 6 of 8 change places
                uint16_t *to = &s_x[wave][i][t][lane / 4 * 4 + lane % 2 * 2 + lane / 2 % 2];
                to[0] = (uint16_t)p[t], to[64] = (uint16_t)(p[t] >> 16);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < PF; ++i) {
            uint32_t d[1][4];
            w[i].codes(0, d[0]);
#pragma unroll
            for (int step = 0; step < 4; step += SPG) {
                bf16x8 xo[SPG][1][PARTS];
#pragma unroll
                for (int s = 0; s < SPG; ++s)
#pragma unroll
                    for (int t = 0; t < PARTS; ++t)
                        xo[s][0][t] = as_bf16x8(*(const u32x4 *)&s_x[wave][i][t][(step + s) * 32 + quad * 8]);
                q4_unit<G, 1, 1, PARTS, SPG>(w[i], d, step, xo, acc);
            }
        }
    }
    if (r == 0) s_o[wave][quad] = acc[0][0];
    __syncthreads();
    if (threadIdx.x < 16 && row0 + threadIdx.x < a.s.rows) {
        float v = 0.f;
        for (int k = 0; k < W; ++k) v += ((const float *)s_o[k])[threadIdx.x];
        q4_store(a, v, row0 + threadIdx.x, 0);
    }
}

// More vectors.  A workgroup computes 16 MT rows for 16 NT vectors; its waves take chunks in turn and
// are joined at the end.  A wave keeps STAGE columns of x at a time in its own part of LDS, so that
// the main loop has no barrier; the next stage's x is asked for before weights, which come from
// farther, so that waiting for x leaves weights of two chunks in flight.
//  * Rows of x are loaded 16 bytes at a time at whatever alignment; what the last load of a row takes
//    past the vectors goes to columns that no output has.
//  * Transposing LDS reads give a lane 4 rows of one column.  Rows of 64 elements are twisted (32-byte
//    pieces exchanged by bits 1 and 3 of the row): the rows that one read touches lay in the same banks.
template <typename X, int NT> constexpr int q4_stage() { return sizeof(X) == 4 ? kQ4Chunk / NT : NT == 4 ? 64 : kQ4Chunk; }
template <typename X, int NT, int MT> constexpr int q4_wave_lds() {
    constexpr int stage = q4_stage<X, NT>() * 16 * NT * 2 * q4_parts<X>(), join = 16 * NT * (16 * MT + 4) * 4;
    return stage > join ? stage : join;
}
//  * ODD: an odd number of bf16 vectors, all in one tile.  Every other row then begins in the middle of
//    a 32-bit word, where loads are slow (4096 x 4096, 7 vectors 8.6 us, 8 vectors 5.5).  They are made
//    from the word's beginning, one element early, and shifted when stored; what a lane lacks at its
//    end is in the first word of the next lane (6.1 us; 8000 x 8000, 3 vectors 16.6 -> 13.0).
template <typename X, int G, int NT, int MT, bool ODD>
__global__ __launch_bounds__(64 * kQ4Waves, 2) void k_q4(Q4Args a) {
    constexpr int PARTS = q4_parts<X>(), STAGE = q4_stage<X, NT>(), WLDS = q4_wave_lds<X, NT, MT>();
    constexpr int RS = 16 * NT, PLANE = STAGE * RS, VE = 16 / sizeof(X), NV = PLANE / VE / 64;   // loads of a lane and stage
    constexpr int US = G == 32 || STAGE == 32 || NT * PARTS > 4 ? 1 : 2; // steps of a unit: their x operands are held in registers
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, quad = lane / 16;
    const int cols = a.s.cols, B = a.batch, W = a.waves, total = cols * B;
    const int64_t row0 = (int64_t)blockIdx.x * (16 * MT);
    const Q4Lane<MT> at(a, row0, r, quad);
    const int c0 = blockIdx.y * RS, nc = min(RS, B - c0);
    uint16_t *mine = (uint16_t *)(lds + wave * WLDS);
    const int n_chunks = (cols + kQ4Chunk - 1) / kQ4Chunk;
    auto twist = [](int row) { return NT == 4 ? (row & 2) << 3 | (row & 8) << 2 : 0; };   // in elements

    // The lane's loads: columns my_k + i * KI of a stage, vectors from my_c on.  They are clamped to x
    // rather than left out (a branch around them would wait for them), and what lies past the end is
    // mended before it is stored: columns past the last are 0, a load that would end past x has begun
    // earlier and is shifted.
    constexpr int KI = 64 * VE / RS;
    const int my_k = lane * VE / RS, my_c = lane * VE % RS;
    const bool tiny = total < VE;     // not one load: read element by element when stored
    const uint8_t *from = tiny ? a.codes : (const uint8_t *)a.x;
    const uint32_t last = tiny ? 0 : (uint32_t)(total - VE) * (uint32_t)sizeof(X), 
                   lane_at = ((uint32_t)my_k * (uint32_t)B + (uint32_t)(c0 + (my_c < nc ? my_c : 0))) * (uint32_t)sizeof(X) &
                             (ODD ? ~3u : ~0u);
    u32x4 v[NV];
    auto load = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            __builtin_memcpy(&v[i], from + min(lane_at + (uint32_t)(k0 + i * KI) * (uint32_t)B * (uint32_t)sizeof(X), last), 16);
        asm volatile("" ::: "memory");   // the loads stay here, a stage ahead of their use
    };
    auto straighten = [&](u32x4 &w) __attribute__((always_inline)) {   // KI is even: a lane's rows are all odd or all even
        const uint32_t next = __builtin_amdgcn_update_dpp(0, w[0], 0x101, 0xf, 0xf, true);   // the next lane's first word
        const int shift = my_k % 2 * 16;
        w = (u32x4){__builtin_amdgcn_alignbit(w[1], w[0], shift), __builtin_amdgcn_alignbit(w[2], w[1], shift),
                    __builtin_amdgcn_alignbit(w[3], w[2], shift), __builtin_amdgcn_alignbit(next, w[3], shift)};
    };
    auto mend = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = k0 + my_k + i * KI;
            const bool in = k < cols && my_c < nc;
            const uint32_t off = lane_at + (uint32_t)(k0 + i * KI) * (uint32_t)B * (uint32_t)sizeof(X);
            if (ODD || tiny) {
                if (ODD) straighten(v[i]);
                if (!in) v[i] = (u32x4){0, 0, 0, 0};
                // ODD: this load or the next lane's has begun earlier (off + 16 may pass 2^32)
                if (in && (!ODD || off > last || last - off < 16)) {
                    alignas(16) X e[VE];
#pragma unroll
                    for (int j = 0; j < VE; ++j) e[j] = my_c + j < nc ? ((const X *)a.x)[k * B + c0 + my_c + j] : (X)0;
                    __builtin_memcpy(&v[i], e, 16);
                }
            } else {
                unsigned __int128 w = __builtin_bit_cast(unsigned __int128, v[i]);
                w = in ? w >> (8 * (off - min(off, last))) : 0;
                v[i] = __builtin_bit_cast(u32x4, w);
            }
        }
    };
    auto store = [&](int k0) __attribute__((always_inline)) {
        if (k0 + STAGE > cols || (int64_t)(k0 + STAGE - 1) * B + c0 + (nc + VE - 1) / VE * VE > total)
            mend(k0);
        else if constexpr (ODD)
#pragma unroll
            for (int i = 0; i < NV; ++i) straighten(v[i]);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = my_k + i * (64 * VE / RS);
            uint16_t *p = mine + k * RS + (my_c ^ twist(k));
            if constexpr (PARTS == 1) {
                *(u32x4 *)p = v[i];
            } else {
                uint32_t q[2][3];
                q4_cut(__uint_as_float(v[i][0]), __uint_as_float(v[i][1]), q[0]);
                q4_cut(__uint_as_float(v[i][2]), __uint_as_float(v[i][3]), q[1]);
#pragma unroll
                for (int t = 0; t < 3; ++t) *(u32x2 *)(p + t * PLANE) = (u32x2){q[0][t], q[1][t]};
            }
        }
    };
    const int lane_row = quad * 8 + r / 4 % 2 * 2 + r / 8;   // of the lane's transposing reads
    int place[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) place[t] = lane_row * RS + ((t * 16 + r % 4 * 4) ^ twist(lane_row));
    auto operand = [&](int k, int t, int part) __attribute__((always_inline)) {
        const uint16_t *p = mine + part * PLANE + k * RS + place[t];
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(p + 4 * RS));
        const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
        return as_bf16x8((u32x4){l.x, l.y, h.x, h.y});
    };
    auto fence = [&]() __attribute__((always_inline)) {   // a wave's LDS operations stay in order; the compiler's too
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    f32x4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[m][t] = (f32x4){0, 0, 0, 0};
    Q4Weights<G, MT> ring[2];
    load(wave * kQ4Chunk);
#pragma unroll
    for (int i = 0; i < 2; ++i) ring[i].load(a, at, min(wave + i * W, n_chunks - 1));
    asm volatile("" ::: "memory");
    auto chunk = [&](int c, Q4Weights<G, MT> &w) __attribute__((always_inline)) {
        uint32_t d[MT][4];
        const Q4Weights<G, MT> now = w;
#pragma unroll
        for (int k = 0; k < kQ4Chunk; k += STAGE) {
            fence();
            store(c * kQ4Chunk + k);
            fence();
            load(k + STAGE < kQ4Chunk ? c * kQ4Chunk + k + STAGE : (c + W) * kQ4Chunk);
            if (k == 0) {
#pragma unroll
                for (int m = 0; m < MT; ++m) now.codes(m, d[m]);
                w.load(a, at, min(c + 2 * W, n_chunks - 1));
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int u = 0; u < STAGE / 32; u += US) {
                bf16x8 xo[US][NT][PARTS];
#pragma unroll
                for (int s = 0; s < US; ++s)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) xo[s][t][p] = operand((u + s) * 32, t, p);
                q4_unit<G, MT, NT, PARTS, US>(now, d, k / 32 + u, xo, acc);
            }
        }
    };
    for (int c = wave; c < n_chunks;) {
        chunk(c, ring[0]);
        if ((c += W) >= n_chunks) break;
        chunk(c, ring[1]);
        c += W;
    }

    // join the waves: [vector][row] of each in LDS
    constexpr int RW = 16 * MT + 4;
    fence();
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) *(f32x4 *)((float *)mine + (t * 16 + r) * RW + m * 16 + quad * 4) = acc[m][t];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * MT * RS; i += 64 * W) {
        const int col = i % RS, row = i / RS;
        if (col >= nc || row0 + row >= a.s.rows) continue;
        float sum = 0.f;
        for (int k = 0; k < W; ++k) sum += ((const float *)(lds + k * WLDS))[col * RW + row];
        q4_store(a, sum, row0 + row, c0 + col);
    }
}

template <typename X, int G, int NT, int MT, bool ODD = false>
hipError_t q4_run(Q4Args a, hipStream_t st) {
    if constexpr (sizeof(X) == 2 && !ODD)
        if (a.batch % 2 && a.batch < 16 * NT && (uintptr_t)a.x % 4 == 0) return q4_run<X, G, NT, MT, true>(a, st);
    constexpr int lds = q4_wave_lds<X, NT, MT>();
    if (kQ4Waves * lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)k_q4<X, G, NT, MT, ODD>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 kQ4Waves * lds);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)div_up64(a.s.rows, 16 * MT), (unsigned)((a.batch + 16 * NT - 1) / (16 * NT)));
    k_q4<X, G, NT, MT, ODD><<<grid, 64 * a.waves, a.waves * lds, st>>>(a);
    return hipGetLastError();
}

// Workgroup shapes.  One vector: a wave has four chunks in flight, so no more waves than fill them
// (1024 x 1024 4.3 us with 8 waves, 3.2 with 2).  More: with few row tiles, as many workgroups as make
// one for each CU (1024 x 1024, 64 vectors: 4.2 us in 16-vector tiles, 5.1 in one of 64; 4096 x 4096
// 22 and 10.5).  Beyond one for each CU, the next would be as long again: two row tiles a wave, which
// also reads x half as often (4200 x 4096, 7 vectors 9.1 -> 8.2 us; 8000 x 8000, 50 vectors 33 -> 23),
// or, where 16 vectors have few chunks, four waves (4099 x 1003, 13 vectors 6.4 -> 5.0, with two row
// tiles 6.4).  With many, both, and a CU holds two workgroups (16384 x 4096, 64 vectors 36 -> 24 us, 16
// vectors 15.7 -> 13.0).
template <typename X, int G>
hipError_t q4_pick(Q4Args a, hipStream_t st) {
    const int n_chunks = (a.s.cols + kQ4Chunk - 1) / kQ4Chunk;
    const int64_t tiles = a.s.rows16 / 16;
    if (a.batch == 1) {
        a.waves = std::min(kQ4Waves, (n_chunks + 3) / 4);
        k_q4_one<X, G><<<(unsigned)tiles, 64 * a.waves, 0, st>>>(a);
        return hipGetLastError();
    }
    a.waves = std::min(kQ4Waves, n_chunks);
    auto groups = [&](int vectors) { return tiles * ((a.batch + vectors - 1) / vectors); };
    if constexpr (sizeof(X) == 4) {   // three operands for each: no more than 16 vectors fit the registers
        const int64_t n = groups(16);
        if (n <= 256) return q4_run<X, G, 1, 1>(a, st);
        if (n <= 512) return q4_run<X, G, 1, 2>(a, st);
        if (n >= 4096) a.waves = std::min(2, n_chunks);   // 16384 x 4096, 61 vectors: 76 us with 8 waves, 57 with 2
        return q4_run<X, G, 1, 4>(a, st);
    } else {
        const int nt = a.batch <= 16 || groups(16) <= 256 ? 1 : a.batch <= 32 || groups(32) <= 256 ? 2 : 4;
        const int64_t n = groups(16 * nt);
        const bool most = n >= (nt == 1 ? 1024 : 512), few = nt == 1 && n_chunks < 16;
        const bool many = most || (n > 256 && !few);
        if (most || (n > 256 && few)) a.waves = std::min(4, n_chunks);
        if (nt == 1) return many ? q4_run<X, G, 1, 2>(a, st) : q4_run<X, G, 1, 1>(a, st);
        if (nt == 2) return many ? q4_run<X, G, 2, 2>(a, st) : q4_run<X, G, 2, 1>(a, st);
        return many ? q4_run<X, G, 4, 2>(a, st) : q4_run<X, G, 4, 1>(a, st);
    }
}

template <typename X>
hipError_t q4_linear(const Q4Args &a, hipStream_t st) {
    return a.s.group == 32 ? q4_pick<X, 32>(a, st) : a.s.group == 64 ? q4_pick<X, 64>(a, st) : q4_pick<X, 128>(a, st);
}

hipError_t q4_linear_bf16(const Q4Args &a, hipStream_t st);
hipError_t q4_linear_f32(const Q4Args &a, hipStream_t st);

}  // namespace bsp
