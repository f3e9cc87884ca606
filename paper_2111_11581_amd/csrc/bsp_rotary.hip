// Rotary positions, with norms of heads in the same pass and the write of keys and values into a
// paged cache.  Queries, keys and values are read once and written once; norm and rotation are in fp32 and rounded once.
// A prompt of 4097 tokens of 32 + 8 heads of 128 dimensions, 101 MB, takes 26.7 us in vectors (3.8 TB/s) and 29.4 with norms,
// where pairs are neighbours 28.6 and 32.3, and 66 feature-major (through LDS, a head at a time).  Angles come before the
// first read of a head, but take no time that shows: with 16 of 128 dimensions rotated 28.8 instead of 28.6.  One token takes
// 4.3 and 32 feature-major ones 4.9, of which norms are 0.6: a launch, then positions, angles, heads and sums, one after
// the other.
#include <hip/hip_runtime.h>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"
#include "bsp_paged.h"

namespace bsp {

namespace {

struct Turn {
    float cos, sin;
};
// Cosine and sine of pos * freq.  Whole turns are taken off in fp64: two products and 1 / 2 pi as it is rounded leave the
// angle of a position up to 2^31 within 2^-21 radians and of one up to 2^20 within 2^-32 (freq up to 1).  What fp32
// cannot hold of the rest, in half turns, turns the result by itself.
__device__ __forceinline__ Turn turn(int pos, double freq) {
    double t = pos * freq * 0.15915494309189533577;   // 1 / 2 pi: turns
    t = 2.0 * (t - rint(t));
    const float half = (float)t, rest = (float)(t - half) * 3.14159265358979f;
    float s, c;
    sincospif(half, &s, &c);
    return {c - s * rest, s + c * rest};
}

// Any layout: a wave for some heads of a token, queries, keys, values, one after the other.
template <typename E> __global__ __launch_bounds__(64) void k_rotary(RotaryArgs a, int each) {
    const int i = blockIdx.x, lane = threadIdx.x, D = a.head_dim, half = a.rope.dims / 2, slots = a.heads + 2 * a.kv_heads;
    const int pos = a.pos[i];
    const bool beside = a.rope.layout == BSP_ROPE_INTERLEAVED;
    Turn r[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int p = lane + 64 * j;
        r[j] = p < half && blockIdx.y * each < a.heads + a.kv_heads ? turn(pos, a.freqs[p]) : Turn{1.f, 0.f};
        r[j].cos *= a.rope.factor, r[j].sin *= a.rope.factor;
    }
    int64_t place = -1;
    if ((blockIdx.y + 1) * each > a.heads && a.kv_heads) place = place_of(a.c, a.table, a.rows ? a.rows[i] : i, a.seqs, a.width, pos);
    for (int slot = blockIdx.y * each; slot < min(slots, (int)(blockIdx.y + 1) * each); ++slot) {
        const bool query = slot < a.heads, value = slot >= a.heads + a.kv_heads;
        const int h = query ? slot : slot - a.heads - (value ? a.kv_heads : 0);
        if (!query && place < 0) return;
        const bsp_strides s = query ? a.xs : value ? a.vs : a.ks;
        const E *src = (const E *)(query ? a.x : value ? a.v : a.k) + i * s.seq + h * s.head;
        E *dst = query ? (E *)a.y + i * a.ys.seq + h * a.ys.head : (E *)(value ? a.values : a.keys) + place + h * a.c.head_stride;
        const int64_t from = s.dim, to = query ? a.ys.dim : 1;
        const float *norm = query ? a.x_norm : value ? nullptr : a.k_norm;
        // a lane's pairs, and its dimensions that are passed on: all are read before any is written
        const int pairs = value ? 0 : half, rest = 2 * pairs;
        float x[2][2], z[4];
        E whole[4];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int p = lane + 64 * j, d0 = beside ? 2 * p : p, d1 = beside ? 2 * p + 1 : p + pairs;
            x[j][0] = p < pairs ? to_f32(src[d0 * from]) : 0.f, x[j][1] = p < pairs ? to_f32(src[d1 * from]) : 0.f;
            sum += x[j][0] * x[j][0] + x[j][1] * x[j][1];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = rest + lane + 64 * j;
            whole[j] = d < D ? src[d * from] : (E)0;
            z[j] = to_f32(whole[j]);
            sum += z[j] * z[j];
        }
        float by = 1.f;
        if (norm) {
            for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
            by = 1.f / sqrtf(sum / D + a.eps);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int p = lane + 64 * j, d0 = beside ? 2 * p : p, d1 = beside ? 2 * p + 1 : p + pairs;
            if (p >= pairs) break;
            if (norm) x[j][0] *= by * norm[d0], x[j][1] *= by * norm[d1];
            dst[d0 * to] = from_f32<E>(x[j][0] * r[j].cos - x[j][1] * r[j].sin);
            dst[d1 * to] = from_f32<E>(x[j][1] * r[j].cos + x[j][0] * r[j].sin);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = rest + lane + 64 * j;
            if (d < D) dst[d * to] = norm ? from_f32<E>(z[j] * (by * norm[d])) : whole[j];
        }
    }
}

// Any layout, many tokens: a workgroup has some tokens, whose cosines and sines it works out once, and some of their
// heads, one after the other, through LDS: read and written along what lies side by side, worked on a token a lane.
template <typename E, int MOST> __global__ __launch_bounds__(256) void k_rotary_tile(RotaryArgs a, int each) {
    constexpr int T = MOST == 128 ? 64 : 32, PARTS = 256 / T, PAD = 4 / sizeof(E);   // rows of an odd number of banks
    __shared__ E s_x[T][MOST + PAD];
    __shared__ Turn s_turn[MOST / 2][T];
    __shared__ float s_sum[PARTS][T];
    __shared__ int64_t s_place[T];
    const int D = a.head_dim, pairs = a.rope.dims / 2, t = threadIdx.x, lane = t % 64, wave = t / 64, token = t % T, part = t / T;
    const int i0 = blockIdx.x * T, n = min(T, a.n - i0), slots = a.heads + 2 * a.kv_heads;
    const bool beside = a.rope.layout == BSP_ROPE_INTERLEAVED;
    for (int p = part; p < pairs; p += PARTS) {
        const Turn r = turn(a.pos[i0 + min(token, n - 1)], a.freqs[p]);
        s_turn[p][token] = {r.cos * a.rope.factor, r.sin * a.rope.factor};
    }
    if (a.kv_heads && t < n) {
        const int i = i0 + t;
        s_place[t] = place_of(a.c, a.table, a.rows ? a.rows[i] : i, a.seqs, a.width, a.pos[i]);
    }
    for (int slot = blockIdx.y * each; slot < min(slots, (int)(blockIdx.y + 1) * each); ++slot) {
        const bool query = slot < a.heads, value = slot >= a.heads + a.kv_heads;
        const int h = query ? slot : slot - a.heads - (value ? a.kv_heads : 0);
        const bsp_strides xs = query ? a.xs : value ? a.vs : a.ks;
        const E *src = (const E *)(query ? a.x : value ? a.v : a.k) + i0 * xs.seq + h * xs.head;
        const float *norm = query ? a.x_norm : value ? nullptr : a.k_norm;
        __syncthreads();   // the head before has been written; places
        if (xs.dim == 1) {
            for (int k = wave; k < n; k += 4)
#pragma unroll
                for (int j = 0; j < MOST / 64; ++j)
                    if (lane + 64 * j < D) s_x[k][lane + 64 * j] = src[k * xs.seq + lane + 64 * j];
        } else {
            const E *from = src + min(token, n - 1) * xs.seq;
#pragma unroll 8
            for (int d = part; d < D; d += PARTS) s_x[token][d] = from[d * xs.dim];
        }
        __syncthreads();
        if (norm) {
            float sum = 0.f;
#pragma unroll 4
            for (int d = part; d < D; d += PARTS) {
                const float x = to_f32(s_x[token][d]);
                sum += x * x;
            }
            s_sum[part][token] = sum;
            __syncthreads();
        }
        if (!value && token < n) {
            float by = 1.f;
            if (norm) {
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < PARTS; ++k) sum += s_sum[k][token];
                by = 1.f / sqrtf(sum / D + a.eps);
            }
#pragma unroll 4
            for (int p = part; p < pairs; p += PARTS) {
                const int d0 = beside ? 2 * p : p, d1 = beside ? d0 + 1 : p + pairs;
                float x = to_f32(s_x[token][d0]), y = to_f32(s_x[token][d1]);
                if (norm) x *= by * norm[d0], y *= by * norm[d1];
                const Turn r = s_turn[p][token];
                s_x[token][d0] = from_f32<E>(x * r.cos - y * r.sin), s_x[token][d1] = from_f32<E>(y * r.cos + x * r.sin);
            }
            if (norm)
                for (int d = 2 * pairs + part; d < D; d += PARTS) s_x[token][d] = from_f32<E>(to_f32(s_x[token][d]) * (by * norm[d]));
        }
        __syncthreads();
        if (!query || a.ys.dim == 1) {
            E *to = query ? (E *)a.y + i0 * a.ys.seq + h * a.ys.head : (E *)(value ? a.values : a.keys) + h * a.c.head_stride;
            for (int k = wave; k < n; k += 4) {
                const int64_t at = query ? k * a.ys.seq : s_place[k];
                if (!query && at < 0) continue;
#pragma unroll
                for (int j = 0; j < MOST / 64; ++j)
                    if (lane + 64 * j < D) to[at + lane + 64 * j] = s_x[k][lane + 64 * j];
            }
        } else if (token < n) {
            E *to = (E *)a.y + (i0 + token) * a.ys.seq + h * a.ys.head;
#pragma unroll 8
            for (int d = part; d < D; d += PARTS) to[d * a.ys.dim] = s_x[token][d];
        }
    }
}

// Heads whose dimensions lie side by side in 16-byte vectors, of which a lane has two: the two halves of its pairs, or
// two neighbours; past the rotated dimensions two that are passed on.  A workgroup has some tokens, whose cosines
// and sines it works out once, and some of their heads, one after the other.  Bound by reading and writing.
struct Rows {
    int lanes_log2, tokens_log2;   // lanes of a head, tokens of a workgroup
    int each;                      // heads of a workgroup that are worked on at a time
};
template <typename E, bool BESIDE> __global__ __launch_bounds__(256) void k_rotary_rows(RotaryArgs a, Rows w) {
    constexpr int VE = 16 / sizeof(E), AHEAD = 4;
    __shared__ Turn s_turn[16 * 128];
    const int D = a.head_dim, pairs = a.rope.dims / 2, t = threadIdx.x;
    const int lane = t & ((1 << w.lanes_log2) - 1), group = t >> w.lanes_log2, token = group & ((1 << w.tokens_log2) - 1);
    const int i0 = blockIdx.x << w.tokens_log2, i = i0 + token, slots = a.heads + 2 * a.kv_heads;
    for (int p = t; p < pairs << w.tokens_log2; p += 256) {
        const int k = p / pairs, at = p - k * pairs;
        Turn r = {1.f, 0.f};
        if (i0 + k < a.n) r = turn(a.pos[i0 + k], a.freqs[at]);
        s_turn[p] = {r.cos * a.rope.factor, r.sin * a.rope.factor};
    }
    // the lane's vectors, or none
    const int rotated = a.rope.dims / VE, vectors = D / VE;
    int first, second;
    bool turned;
    if (BESIDE) {
        first = 2 * lane, second = first + 1, turned = first < rotated;
    } else {
        turned = 2 * lane < rotated;
        first = turned ? lane : 2 * lane, second = turned ? lane + rotated / 2 : first + 1;
    }
    // Of an odd number of rotated vectors the last one's neighbour is passed on: its bits, as its values times 1 and
    // 0 would let an Inf or a NaN reach the other dimension of a pair.
    const bool passed = BESIDE && turned && second >= rotated;
    const bool in = i < a.n, has[2] = {in && first < vectors, in && second < vectors};
    const int d[2] = {min(first, vectors - 1) * VE, min(second, vectors - 1) * VE};
    int64_t place = -1;
    if (a.kv_heads && in) place = place_of(a.c, a.table, a.rows ? a.rows[i] : i, a.seqs, a.width, a.pos[i]);
    __syncthreads();
    // cosines and sines: of pairs of dimensions j of both vectors, or of neighbours in each
    float c[VE], sn[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) {
        const int p = BESIDE ? first * (VE / 2) + j : first * VE + j;
        const Turn r = turned && p < pairs ? s_turn[token * pairs + p] : Turn{1.f, 0.f};
        c[j] = r.cos, sn[j] = r.sin;
    }
    const int h0 = blockIdx.y * w.each * (256 >> (w.lanes_log2 + w.tokens_log2)) + (group >> w.tokens_log2);
    const int step = 256 >> (w.lanes_log2 + w.tokens_log2);
    for (int k0 = 0; k0 < w.each; k0 += AHEAD) {
        u32x4 v[AHEAD][2];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int h = min(h0 + (k0 + k) * step, slots - 1), at = min(i, a.n - 1);
            const E *src = h < a.heads ? (const E *)a.x + at * a.xs.seq + h * a.xs.head
                           : h < a.heads + a.kv_heads ? (const E *)a.k + at * a.ks.seq + (h - a.heads) * a.ks.head
                                                      : (const E *)a.v + at * a.vs.seq + (h - a.heads - a.kv_heads) * a.vs.head;
            if (k0 + k < w.each) v[k][0] = *(const u32x4 *)(src + d[0]), v[k][1] = *(const u32x4 *)(src + d[1]);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int h = h0 + (k0 + k) * step;
            const bool query = h < a.heads, value = h >= a.heads + a.kv_heads, go = k0 + k < w.each && h < slots && (query || place >= 0);
            E *dst = query ? (E *)a.y + i * a.ys.seq + h * a.ys.head
                           : (E *)(value ? a.values : a.keys) + place + (h - a.heads - (value ? a.kv_heads : 0)) * a.c.head_stride;
            const float *norm = query ? a.x_norm : value ? nullptr : a.k_norm;
            if (!value && (norm || turned)) {
                float x[2][VE];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        if constexpr (sizeof(E) == 4) {
                            const uint32_t bits = v[k][s][j];
                            x[s][j] = __uint_as_float(bits);
                        } else {
                            const uint32_t bits = v[k][s][j / 2];
                            x[s][j] = __uint_as_float(j % 2 ? bits & 0xffff0000u : bits << 16);
                        }
                    }
                if (norm) {
                    float sum = 0.f;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        float part = 0.f;
#pragma unroll
                        for (int j = 0; j < VE; ++j) part += x[s][j] * x[s][j];
                        sum += has[s] ? part : 0.f;
                    }
                    for (int o = 1; o < 1 << w.lanes_log2; o *= 2) sum += __shfl_xor(sum, o);
                    const float by = 1.f / sqrtf(sum / D + a.eps);
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int j = 0; j < VE; ++j) x[s][j] *= by * norm[d[s] + j];
                }
                if (turned) {
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        if (2 * j / VE == 1 && passed) continue;
                        float *p = BESIDE ? &x[2 * j / VE][2 * j % VE] : &x[0][j], *o = BESIDE ? p + 1 : &x[1][j];
                        const float y = *p * c[j] - *o * sn[j];
                        *o = *o * c[j] + *p * sn[j], *p = y;
                    }
                }
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (s == 1 && passed && !norm) continue;
                        if constexpr (sizeof(E) == 4) v[k][s][j] = __float_as_uint(x[s][j]);
                        else v[k][s][j] = pack_bf16(x[s][2 * j], x[s][2 * j + 1]);
                    }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (go && has[s]) *(u32x4 *)(dst + d[s]) = v[k][s];
        }
    }
}

// Whether rows of heads begin at 16 bytes.
bool in_vectors(const void *p, const bsp_strides &s, int esize) {
    return s.dim == 1 && (uintptr_t)p % 16 == 0 && s.seq * esize % 16 == 0 && s.head * esize % 16 == 0;
}

// Tiles are for what lies along the tokens, from so many tokens on: 256 tokens of 48 heads take 13.8 us and by waves 16.1,
// 4097 tokens 66 and 203, but 96 tokens 13.6 and 8.5.  Along the dimensions waves read as well: 4097 tokens of 80
// dimensions, 40 of them rotated, 67 in tiles and 70, of 256 dimensions 64 and 31.
constexpr int kTile = 192;
// Waves by which the heads of a token are shared, each working the angles out: those 4097 tokens 70 us, with half as many
// waves 82, with one for each head 85; 1000 tokens 20.2, 20.1 and 23.0.
constexpr int kWaves = 16384;

template <typename E> hipError_t run(const RotaryArgs &a, hipStream_t st) {
    constexpr int VE = 16 / sizeof(E);
    const int slots = a.heads + 2 * a.kv_heads, esize = sizeof(E);
    const bool beside = a.rope.layout == BSP_ROPE_INTERLEAVED;
    const bool rows = a.head_dim % VE == 0 && a.rope.dims % (beside ? VE : 2 * VE) == 0 && in_vectors(a.x, a.xs, esize) &&
                      in_vectors(a.y, a.ys, esize) && (!a.kv_heads || (in_vectors(a.k, a.ks, esize) && in_vectors(a.v, a.vs, esize)));
    if (!rows && (a.xs.dim == 1 || a.n < kTile)) {
        const int each = (int)std::max<int64_t>(1, std::min<int64_t>(slots, (int64_t)a.n * slots / kWaves));
        k_rotary<E><<<dim3(a.n, (slots + each - 1) / each), 64, 0, st>>>(a, each);
        return hipGetLastError();
    }
    if (!rows) {
        const bool wide = a.head_dim > 128;
        const int tiles = (a.n + (wide ? 31 : 63)) / (wide ? 32 : 64), each = std::max(1, std::min(slots, (int)((int64_t)tiles * slots / 768)));
        const dim3 grid(tiles, (slots + each - 1) / each);
        if (wide) k_rotary_tile<E, 256><<<grid, 256, 0, st>>>(a, each);
        else k_rotary_tile<E, 128><<<grid, 256, 0, st>>>(a, each);
        return hipGetLastError();
    }
    // A workgroup's groups of lanes go to up to 16 tokens, then to heads; few tokens leave each workgroup one head of a
    // group, many all heads, for which the angles are worked out once.
    Rows w;
    w.lanes_log2 = 0;
    while (2 << w.lanes_log2 < a.head_dim / VE) ++w.lanes_log2;
    w.tokens_log2 = 0;
    while (w.tokens_log2 < 4 && w.lanes_log2 + w.tokens_log2 < 6 && a.n >= 32 << w.tokens_log2) ++w.tokens_log2;
    const int per = 256 >> (w.lanes_log2 + w.tokens_log2), all = (slots + per - 1) / per;
    const int tokens = (a.n + (1 << w.tokens_log2) - 1) >> w.tokens_log2;
    w.each = std::max(1, std::min(all, (int)((int64_t)tokens * all / 1024)));
    const dim3 grid(tokens, (all + w.each - 1) / w.each);
    if (beside) k_rotary_rows<E, true><<<grid, 256, 0, st>>>(a, w);
    else k_rotary_rows<E, false><<<grid, 256, 0, st>>>(a, w);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t st) {
    return a.dtype == BSP_F32 ? run<float>(a, st) : run<uint16_t>(a, st);
}

}  // namespace bsp
