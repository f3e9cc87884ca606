// Attention of one new token over a paged cache, and the write of its key and value.
//
// k_attn reads every key and value once, straight from memory into the registers of the matrix
// instructions, and never through LDS:
//  * scores, transposed: rows are tokens, columns the (up to 16) query heads that share the key
//    head.  The A operand (keys) is 16 bytes of a token per lane as it lies in memory; since a sum
//    over dimensions has no order, queries take the same order.
//  * a lane of the result holds one head's scores of 4 tokens of each tile, which is what the B
//    operand of the next product (tokens x heads) wants, if its tokens are numbered that way.  So
//    probabilities go from one product to the next in place.
//  * outputs, transposed: rows are dimensions, columns heads.  A lane loads VW dimensions of each of
//    its quad's tokens; for bf16 pairs of tokens are interleaved (32 byte permutes for 8 x 8
//    values), dimension j of every lane makes one operand.
// The running maximum and sum of the softmax are kept per head (per lane); the sum of a lane's own
// tokens is added over lanes at the end.  It is bound by reading keys and values: of a CU's cycles,
// at 9 bytes each, a step of 32 tokens of 128 dimensions needs 1820, and its 16 products 256.
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"

namespace bsp {

namespace {

constexpr int kWaves = 4, kTile = 512;   // waves of a workgroup; tokens whose places it keeps in LDS
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

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

// The tokens of a sequence, and how many parts of `chunk` they make (1 where there are none).
struct Span {
    int first, len, parts;
};
__device__ __forceinline__ Span span_of(const AttnArgs &a, int b, int *row) {
    *row = a.rows ? a.rows[b] : b;
    Span s;
    s.len = (unsigned)*row < (unsigned)a.seqs ? a.lens[*row] : 0;
    s.len = max(0, (int)min((int64_t)s.len, (int64_t)a.width * a.c.page_size));
    s.first = a.window && s.len > a.window ? s.len - a.window : 0;
    s.parts = max(1, (int)(((unsigned)(s.len - s.first) + a.chunk - 1) / a.chunk));
    return s;
}

// What a wave loads and multiplies in one step, for head_dim up to DP.
template <typename E, int DP> struct Step;

template <int DP> struct Step<uint16_t, DP> {
    static constexpr int TOK = 32, NK = DP / 32, VW = DP == 64 ? 4 : 8, NV = DP / (16 * VW);
    typedef uint32_t VRaw __attribute__((ext_vector_type(VW / 2)));
    uint4 q[NK];
    uint4 k[2][NK];
    VRaw v[8][NV];

    __device__ __forceinline__ void load_q(const uint16_t *p, int64_t stride, bool on, int quad, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = c * 32 + quad * 8 + 2 * i;
                w[i] = on && d < D ? p[d * stride] | (uint32_t)p[(d + 1) * stride] << 16 : 0u;
            }
            q[c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // ko: places of tokens l % 16 and 16 + l % 16; vo: of tokens 4 quad + i and 16 + 4 quad + i
    template <bool FULL>
    __device__ __forceinline__ void load(const uint16_t *keys, const uint16_t *values, const int64_t *ko, const int64_t *vo,
                                         int quad, int r, int D) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const int d = c * 32 + quad * 8;
                const bool in = FULL || d < D;
                k[t][c] = *(const uint4 *)(keys + max(ko[t], (int64_t)0) + (in ? d : 0));
                if (!in) k[t][c] = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int h = 0; h < NV; ++h) {
                const int d = h * 16 * VW + r * VW;
                v[i][h] = *(const VRaw *)(values + max(vo[i], (int64_t)0) + (FULL || d < D ? d : 0));
            }
    }
    __device__ __forceinline__ void clear_v(const int64_t *vo) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (vo[i] < 0)
#pragma unroll
                for (int h = 0; h < NV; ++h) v[i][h] = (VRaw)0;
    }
    __device__ __forceinline__ void scores(float *s) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 c4 = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < NK; ++c)
                c4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k[t][c]), as_bf16x8(q[c]), c4, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * t + i] = c4[i];
        }
    }
    // Probabilities are rounded to bf16 here: their product runs on bf16 operands.
    __device__ __forceinline__ void outputs(const float *p, f32x4 (*acc)[VW]) const {
        const uint4 b = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7]));
#pragma unroll
        for (int h = 0; h < NV; ++h)
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                const uint32_t sel = j % 2 ? 0x07060302u : 0x05040100u;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(v[2 * i + 1][h][j / 2], v[2 * i][h][j / 2], sel);
                acc[h][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(make_uint4(w[0], w[1], w[2], w[3])),
                                                                    as_bf16x8(b), acc[h][j], 0, 0, 0);
            }
    }
};

template <int DP> struct Step<float, DP> {
    static constexpr int TOK = 16, NK = DP / 16, VW = 4, NV = DP / 64;
    f32x4 q[NK];
    f32x4 k[NK];
    f32x4 v[4][NV];

    __device__ __forceinline__ void load_q(const float *p, int64_t stride, bool on, int quad, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = c * 16 + quad * 4 + i;
                q[c][i] = on && d < D ? p[d * stride] : 0.f;
            }
    }
    template <bool FULL>
    __device__ __forceinline__ void load(const float *keys, const float *values, const int64_t *ko, const int64_t *vo,
                                         int quad, int r, int D) {
#pragma unroll
        for (int c = 0; c < NK; ++c) {
            const int d = c * 16 + quad * 4;
            const bool in = FULL || d < D;
            k[c] = *(const f32x4 *)(keys + max(ko[0], (int64_t)0) + (in ? d : 0));
            if (!in) k[c] = (f32x4){0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < NV; ++h) {
                const int d = h * 64 + r * 4;
                v[i][h] = *(const f32x4 *)(values + max(vo[i], (int64_t)0) + (FULL || d < D ? d : 0));
            }
    }
    __device__ __forceinline__ void clear_v(const int64_t *vo) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (vo[i] < 0)
#pragma unroll
                for (int h = 0; h < NV; ++h) v[i][h] = (f32x4){0, 0, 0, 0};
    }
    __device__ __forceinline__ void scores(float *s) const {
        f32x4 c4 = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < NK; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) c4 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][i], q[c][i], c4, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = c4[i];
    }
    __device__ __forceinline__ void outputs(const float *p, f32x4 (*acc)[VW]) const {
#pragma unroll
        for (int h = 0; h < NV; ++h)
#pragma unroll
            for (int j = 0; j < VW; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[h][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][h][j], p[i], acc[h][j], 0, 0, 0);
    }
};

// A workgroup: one part of a sequence's tokens, for up to 16 query heads of one key head.  Its waves
// take the steps in turn and are joined through LDS; a sequence of one part is finished here, others
// leave (maximum, sum) and outputs of their parts in the workspace.
template <typename E, int DP, bool FULL>
__global__ __launch_bounds__(64 * kWaves, DP == 256 ? 1 : 2) void k_attn(AttnArgs a) {
    typedef Step<E, DP> St;
    constexpr int TOK = St::TOK, TT = TOK / 4, NT = TOK / 16, VW = St::VW, NV = St::NV, ROW = DP + 4;
    __shared__ int64_t place[kTile];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16], s_o[2][16][ROW];

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, quad = lane / 16, D = a.c.head_dim;
    const int part = blockIdx.x % a.splits, unit = blockIdx.x / a.splits;   // unit: (sequence, key head, head group)
    const int hg = unit % a.head_groups, bj = unit / a.head_groups, j = bj % a.c.kv_heads, b = bj / a.c.kv_heads;
    int row;
    const Span sp = span_of(a, b, &row);
    if (part >= sp.parts) return;
    const int from = sp.first + part * a.chunk, to = min(sp.len, from + a.chunk);
    const int heads = min(16, a.group - hg * 16), h0 = j * a.group + hg * 16;

    St st;
    st.load_q((const E *)a.q + b * a.qs.seq + (h0 + min(r, heads - 1)) * a.qs.head, a.qs.dim, r < heads, quad, D);
    f32x4 acc[NV][VW];
#pragma unroll
    for (int h = 0; h < NV; ++h)
#pragma unroll
        for (int i = 0; i < VW; ++i) acc[h][i] = (f32x4){0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    const float scale = a.scale * kLog2e;
    const int32_t *table = a.table + (int64_t)row * a.width;

    for (int base = from; base < to; base += kTile) {
        const int n = min(kTile, to - base), padded = (n + TOK - 1) / TOK * TOK;
        if (base > from) __syncthreads();   // places of the tile before are no longer read
        for (int t = threadIdx.x; t < padded; t += 64 * kWaves) {
            int64_t at = -1;
            if (t < n) {
                uint32_t slot;
                const int page = page_of(a.c, table, (uint32_t)(base + t), &slot);
                if (page >= 0) at = page * a.c.page_stride + slot * a.c.slot_stride + j * a.c.head_stride;
            }
            place[t] = at;
        }
        __syncthreads();
        for (int s0 = wave * TOK; s0 < padded; s0 += kWaves * TOK) {
            int64_t ko[NT], vo[TT];
            bool all = true;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                ko[t] = place[s0 + 16 * t + r];
                all = all && ko[t] >= 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) vo[4 * t + i] = place[s0 + 16 * t + 4 * quad + i];
            }
            st.template load<FULL>((const E *)a.keys, (const E *)a.values, ko, vo, quad, r, D);
            float s[TT];
            st.scores(s);
            const bool whole = __all(all);
            float top = m;
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                s[i] *= scale;
                if (!whole && vo[i] < 0) s[i] = -INFINITY;
                top = fmaxf(top, s[i]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float ref = top == -INFINITY ? 0.f : top;
            const float keep = __builtin_amdgcn_exp2f(m - ref);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                s[i] = __builtin_amdgcn_exp2f(s[i] - ref);
                sum += s[i];
            }
            l = l * keep + sum;
            m = top;
            if (!whole) st.clear_v(vo);
            if (__any(keep != 1.f))
#pragma unroll
                for (int h = 0; h < NV; ++h)
#pragma unroll
                    for (int i = 0; i < VW; ++i) acc[h][i] *= keep;
            st.outputs(s, acc);
        }
    }

    // join the waves: all on the common maximum, then 2 and 3 onto 0 and 1
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (quad == 0) s_m[wave][r] = m, s_l[wave][r] = l;
    __syncthreads();
    float top = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    for (int turn = 0; turn < 2; ++turn) {
        if (wave / 2 == 1 - turn && r < heads)
#pragma unroll
            for (int h = 0; h < NV; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < VW; v += 4) {
                        f32x4 *o = (f32x4 *)&s_o[wave % 2][r][h * 16 * VW + (quad * 4 + i) * VW + v];
                        f32x4 x = {acc[h][v][i], acc[h][v + 1][i], acc[h][v + 2][i], acc[h][v + 3][i]};
                        x *= f;
                        *o = turn ? *o + x : x;
                    }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < heads * DP; i += 64 * kWaves) {
        const int h = i / DP, d = i % DP;
        if (d >= D) continue;
        float mm = s_m[0][h], sum = 0.f;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, s_m[w][h]);
        const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += s_l[w][h] * __builtin_amdgcn_exp2f(s_m[w][h] - ref);
        const float o = s_o[0][h][d] + s_o[1][h][d];
        const int64_t bh = (int64_t)b * a.heads + h0 + h;
        if (sp.parts == 1) {
            E *y = (E *)a.y + b * a.ys.seq + (h0 + h) * a.ys.head + d * a.ys.dim;
            *y = from_f32<E>(sum == 0.f ? 0.f : o / sum);
            if (d == 0 && a.lse) a.lse[bh] = (ref + log2f(sum)) * kLn2;
        } else {
            float *ml = (float *)a.workspace, *out = ml + 2 * (int64_t)a.batch * a.heads * a.splits;
            out[(bh * a.splits + part) * D + d] = o;
            if (d == 0) ml[(bh * a.splits + part) * 2] = mm, ml[(bh * a.splits + part) * 2 + 1] = sum;
        }
    }
}

// Joins the parts of a sequence's query head: a workgroup each, a thread a dimension of every
// 256 / DP-th part.
constexpr int kMaxSplits = 256;
template <typename E, int DP>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
    __shared__ float s_w[kMaxSplits], s_red[8], s_o[256];
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.heads), h = (int)(bh - (int64_t)b * a.heads), t = threadIdx.x, D = a.c.head_dim;
    int row;
    const Span sp = span_of(a, b, &row);
    if (sp.parts == 1) return;
    const float *ml = (const float *)a.workspace + bh * a.splits * 2;
    const float *o = (const float *)a.workspace + 2 * (int64_t)a.batch * a.heads * a.splits + bh * a.splits * D;
    const float m = t < sp.parts ? ml[2 * t] : -INFINITY, l = t < sp.parts ? ml[2 * t + 1] : 0.f;
    float top = m;
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    if (t % 64 == 0) s_red[t / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    const float ref = top == -INFINITY ? 0.f : top, w = __builtin_amdgcn_exp2f(m - ref);
    float sum = l * w;
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (t % 64 == 0) s_red[4 + t / 64] = sum;
    s_w[t] = w;
    __syncthreads();
    sum = (s_red[4] + s_red[5]) + (s_red[6] + s_red[7]);
    constexpr int G = 256 / DP;
    const int d = t % DP, g = t / DP;
    float v = 0.f;
    if (d < D)
        for (int p = g; p < sp.parts; p += G) v += o[(int64_t)p * D + d] * s_w[p];
    s_o[t] = v;
    __syncthreads();
    if (t >= D) return;
#pragma unroll
    for (int i = 1; i < G; ++i) v += s_o[t + i * DP];
    E *y = (E *)a.y + b * a.ys.seq + h * a.ys.head + t * a.ys.dim;
    *y = from_f32<E>(sum == 0.f ? 0.f : v / sum);
    if (t == 0 && a.lse) a.lse[bh] = (ref + log2f(sum)) * kLn2;
}

// How the tokens are split: about `kTarget` workgroups if all sequences were as long as they may be,
// parts of at least kMinChunk tokens (two steps a wave).
constexpr int kTarget = 1024, kMinChunk = 256;
int units_of(const CacheArgs &c, int batch, int heads) {
    return batch * c.kv_heads * ((heads / c.kv_heads + 15) / 16);
}
int most_splits(const CacheArgs &c, int batch, int heads) {
    return std::min(kMaxSplits, std::max(1, kTarget / std::max(1, units_of(c, batch, heads))));
}

template <typename E, int DP, bool FULL>
hipError_t run(const AttnArgs &a, hipStream_t st) {
    k_attn<E, DP, FULL><<<units_of(a.c, a.batch, a.heads) * a.splits, 64 * kWaves, 0, st>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
    k_attn_join<E, DP><<<a.batch * a.heads, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <typename E>
hipError_t run(const AttnArgs &a, hipStream_t st) {
    const int D = a.c.head_dim;
    if (D <= 64) return D == 64 ? run<E, 64, true>(a, st) : run<E, 64, false>(a, st);
    if (D <= 128) return D == 128 ? run<E, 128, true>(a, st) : run<E, 128, false>(a, st);
    return D == 256 ? run<E, 256, true>(a, st) : run<E, 256, false>(a, st);
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

// (maximum, sum) and head_dim outputs of every part of every query head
int64_t attention_workspace(const CacheArgs &c, int batch, int heads, int width) {
    const int64_t most = std::min<int64_t>(most_splits(c, batch, heads), div_up64((int64_t)width * c.page_size, kMinChunk));
    return most <= 1 ? 0 : (int64_t)batch * heads * most * (c.head_dim + 2) * 4;
}

hipError_t launch_attention(AttnArgs a, hipStream_t st) {
    int64_t tokens = (int64_t)a.width * a.c.page_size;
    if (a.window) tokens = std::min<int64_t>(tokens, a.window);
    const int64_t most = most_splits(a.c, a.batch, a.heads);
    a.chunk = (int)std::max<int64_t>(kMinChunk, div_up64(div_up64(tokens, most), 128) * 128);
    a.splits = (int)std::max<int64_t>(1, div_up64(tokens, a.chunk));
    a.head_groups = (a.group + 15) / 16;
    return a.c.dtype == BSP_F32 ? run<float>(a, st) : run<uint16_t>(a, st);
}

}  // namespace bsp
