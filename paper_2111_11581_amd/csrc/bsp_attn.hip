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
// at 9 bytes each, a step of 32 tokens of 128 dimensions needs 1820, and its 24 products 384 (131072
// tokens of 8 key heads, 537 MB: 88 us; 32 sequences of up to 2048 tokens, 134 MB: 36; a few short
// sequences: the latency of length, entry, key, value and join, 4.4 for 77 tokens).
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"

namespace bsp {

namespace {

constexpr int kWaves = 4, kTile = 1024;   // waves of a workgroup; tokens whose places it keeps in LDS
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Page of token t of a sequence, or -1 where the entry holds nothing.
__device__ __forceinline__ int page_of(const CacheArgs &c, const int32_t *row, uint32_t t, uint32_t *slot) {
    const uint32_t e = fdiv(t, c.div_page);
    *slot = t - e * (uint32_t)c.page_size;
    const int p = row[e];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
}

// A thread copies elements of a token's key or value.  Bound by the latency of position, entry and
// store, one after the other; the elements are read meanwhile (32 tokens of 1024 elements 4.0 us, 4.9
// where they were read last; an empty kernel 3).
template <typename E>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
    constexpr int kAhead = 4;
    const int i = blockIdx.x, dims = a.c.kv_heads * a.c.head_dim;
    const E *src = (const E *)(blockIdx.y ? a.v : a.k);
    const bsp_strides s = blockIdx.y ? a.vs : a.ks;
    const int row = a.rows ? a.rows[i] : i, pos = a.pos[i];
    auto element = [&](int j) {
        const int h = j / a.c.head_dim, d = j - h * a.c.head_dim;
        return src[i * s.seq + h * s.head + d * s.dim];
    };
    E ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ahead[k] = element(min((int)threadIdx.x + k * 256, dims - 1));
    if ((unsigned)row >= (unsigned)a.seqs || pos < 0) return;
    if (pos >= (int64_t)a.width * a.c.page_size) return;
    uint32_t slot;
    const int page = page_of(a.c, a.table + (int64_t)row * a.width, (uint32_t)pos, &slot);
    if (page < 0) return;
    E *dst = (E *)(blockIdx.y ? a.values : a.keys) + page * a.c.page_stride + slot * a.c.slot_stride;
    auto put = [&](int j, E v) {
        const int h = j / a.c.head_dim;
        dst[h * a.c.head_stride + (j - h * a.c.head_dim)] = v;
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if ((int)threadIdx.x + k * 256 < dims) put(threadIdx.x + k * 256, ahead[k]);
    for (int j = threadIdx.x + kAhead * 256; j < dims; j += 256) put(j, element(j));
}

__device__ __forceinline__ int row_of(const AttnArgs &a, int b) { return a.rows ? a.rows[b] : b; }
__device__ __forceinline__ int len_of(const AttnArgs &a, int row) {
    const int len = (unsigned)row < (unsigned)a.seqs ? a.lens[row] : 0;
    return max(0, (int)min((int64_t)len, (int64_t)a.width * a.c.page_size));
}
// The tokens that a sequence attends to, and their number in blocks of 32.
constexpr int kBlock = 32;
struct Span {
    int row, first, len, blocks;
};
__device__ __forceinline__ Span span_of(const AttnArgs &a, int row, int len) {
    Span s;
    s.row = row, s.len = len;
    s.first = a.window && s.len > a.window ? s.len - a.window : 0;
    s.blocks = (int)(((unsigned)(s.len - s.first) + kBlock - 1) / kBlock);
    return s;
}

// How the work is shared out, when sequences are split.  A unit is a sequence's tokens for one head
// group.  All units, in a row, are cut into equal shares, one for each workgroup, whatever the lengths
// are.  Share g and unit u meet in at most one segment, number g + u (one of the two grows from each
// segment to the next).  A unit counts
//  * in pieces of 4 blocks, a step of each wave (bf16) or two (fp32), if that gives no more pieces than
//    workgroups; a share is a piece (60 units of 25 fp32 blocks 28 -> 21 us);
//  * else in blocks, and kCost more (what beginning and ending a segment takes: 5 of a segment's 19 us
//    where 17 blocks take 13; without it the workgroups that get many short units take twice as long).
// Every workgroup works the cuts out for itself from the lengths: s_before[b] is the length of a head
// group's units before sequence b, s_len[b] its tokens.
constexpr int kCost = 8, kMinShare = kCost + 8;
constexpr int kMostSeqs = 1024, kMostShares = 512;
struct Cut {
    int size_log2, cost;
    int64_t share, total;
    __device__ __forceinline__ int length(int blocks) const {
        return blocks ? ((blocks - 1) >> size_log2) + 1 + cost : 0;
    }
};
__device__ __forceinline__ Cut cut_up(const AttnArgs &a, int32_t *s_before, int32_t *s_len) {
    constexpr int PER = kMostSeqs / 256;
    __shared__ int s_wave[4];
    const int t = threadIdx.x, lane = t % 64;
    int blocks[PER];
    const int per = (a.batch + 255) / 256;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        blocks[i] = 0;
        if (i < per && t * per + i < a.batch) {
            const int len = len_of(a, row_of(a, t * per + i));
            s_len[t * per + i] = len;
            blocks[i] = span_of(a, 0, len).blocks;
        }
    }
    Cut c = {2, 0, 1, 0};
    for (;;) {
        int sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) sum += c.length(blocks[i]);
        int upto = sum;
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 63) s_wave[t / 64] = upto;
        __syncthreads();
        int before = upto - sum, all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            before += w < t / 64 ? s_wave[w] : 0;
            all += s_wave[w];
        }
        c.total = (int64_t)uni(all) * (a.c.kv_heads * a.head_groups);
        if (!c.cost && c.total > a.shares) {
            c = {0, kCost, 1, 0};
            __syncthreads();   // s_wave has been read
            continue;
        }
        if (c.cost) c.share = max((int64_t)kMinShare, (c.total + a.shares - 1) / a.shares);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (i < per && t * per + i <= a.batch) {
                s_before[t * per + i] = before;
                before += c.length(blocks[i]);
            }
        if (t == 255) s_before[a.batch] = all;   // the last thread's own end is everyone's
        break;
    }
    __syncthreads();
    return c;
}

// ONCE: past the caches.
template <bool ONCE, typename T> __device__ __forceinline__ T fetch(const T *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

// What a wave loads and multiplies in one step, for head_dim up to DP.
template <typename E, int DP> struct Step;

template <int DP> struct Step<uint16_t, DP> {
    static constexpr int TOK = 32, NK = DP / 32, VW = DP == 64 ? 4 : 8, NV = DP / (16 * VW);
    typedef uint32_t VRaw __attribute__((ext_vector_type(VW / 2)));
    u32x4 q[NK];
    u32x4 k[2][NK];
    VRaw v[8][NV];

    __device__ __forceinline__ void load_q(const uint16_t *row, int quad) {
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
    template <bool FULL> __device__ __forceinline__ void scores(float *s, int D) const {
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
    __device__ __forceinline__ void outputs(const float *p, f32x4 (*acc)[VW]) const {
        u32x4 b[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            b[0][i] = pack_bf16(p[2 * i], p[2 * i + 1]);
            b[1][i] = pack_bf16(p[2 * i] - bf16_to_f32(b[0][i]), p[2 * i + 1] - __uint_as_float(b[0][i] & 0xffff0000u));
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
                    acc[h][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(b[i]), acc[h][j], 0, 0, 0);
            }
    }
};

template <int DP> struct Step<float, DP> {
    static constexpr int TOK = 16, NK = DP / 16, VW = 4, NV = DP / 64;
    f32x4 q[NK];
    f32x4 k[NK];
    f32x4 v[4][NV];

    __device__ __forceinline__ void load_q(const float *row, int quad) {
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
    template <bool FULL> __device__ __forceinline__ void scores(float *s, int D) const {
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

// The workspace: maxima and sums, then outputs, of segments' heads; first share and number of segments
// of each unit.
struct Parts {
    float *m, *l, *o;
    int2 *count;
    int heads;
    __device__ __forceinline__ explicit Parts(const AttnArgs &a) : heads(min(16, a.group)) {
        const int64_t units = (int64_t)a.batch * a.c.kv_heads * a.head_groups, n = (a.shares + units) * heads;
        o = (float *)a.workspace, m = o + n * a.c.head_dim, l = m + n;   // of o, 16 bytes at a time are read
        count = (int2 *)(l + n);
    }
    __device__ __forceinline__ int64_t at(int64_t segment, int head) const { return segment * heads + head; }
};

// A workgroup: its share of the work, or (shares 0) a unit: a sequence's tokens for up to 16 query heads
// of one key head.  In a segment its waves take the steps in turn and are joined through LDS; a unit
// of one segment is finished here, others leave (maximum, sum) and outputs of their segments in the
// workspace.
template <typename E, int DP, bool FULL, bool SHARED, bool ONCE>
__global__ __launch_bounds__(64 * kWaves, DP == 256 ? 1 : 2) void k_attn(AttnArgs a) {
    typedef Step<E, DP> St;
    constexpr int TOK = St::TOK, TT = TOK / 4, NT = TOK / 16, VW = St::VW, NV = St::NV, ROW = DP + 4;
    __shared__ int64_t place[kTile];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16], s_o[2][16][ROW];
    __shared__ int32_t s_before[SHARED ? kMostSeqs + 1 : 1], s_len[SHARED ? kMostSeqs : 1];
    __shared__ __attribute__((aligned(16))) E s_q[16][DP + 16 / sizeof(E)];

    const int wave = uni(threadIdx.x / 64), D = a.c.head_dim;
    const int per_seq = a.c.kv_heads * a.head_groups;   // units of a sequence
    int64_t pos = 0, end = 1;
    Cut cut;
    if (SHARED) {
        cut = cut_up(a, s_before, s_len);
        pos = blockIdx.x * cut.share, end = min(pos + cut.share, cut.total);
        // sequences without tokens: no workgroup's work
        for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
            if (uni(s_before[b + 1]) != uni(s_before[b])) continue;
            for (int i = threadIdx.x; i < per_seq; i += 64 * kWaves) Parts(a).count[b * (int64_t)per_seq + i] = make_int2(0, 1);
            for (int i = threadIdx.x; i < a.heads * D; i += 64 * kWaves)
                ((E *)a.y)[b * a.ys.seq + i / D * a.ys.head + i % D * a.ys.dim] = (E)0;
            if (a.lse)
                for (int i = threadIdx.x; i < a.heads; i += 64 * kWaves) a.lse[(int64_t)b * a.heads + i] = -INFINITY;
        }
    }
    while (pos < end) {
    int lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));   // what goes by the lane is worked out again for each segment, not held in registers
    const int r = lane % 16, quad = lane / 16;
    int b, u, from, to;
    bool whole_unit = true;
    int64_t segment = 0;
    Span sp;
    if (SHARED) {
        int lo = 0, hi = a.batch;   // the last sequence that begins at or before pos, which has blocks
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((int64_t)uni(s_before[mid]) * per_seq <= pos) lo = mid; else hi = mid;
        }
        b = lo;
        sp = span_of(a, uni(row_of(a, b)), uni(s_len[b]));
        const int64_t rest = pos - (int64_t)uni(s_before[b]) * per_seq;
        const int length = cut.length(sp.blocks);
        u = uni((int)(rest / length));
        const int off = (int)(rest - (int64_t)u * length), n = (int)min(end - pos, (int64_t)(length - off));
        const int first = max(0, off - cut.cost) << cut.size_log2;   // blocks of the segment
        const int last = min(max(0, off + n - cut.cost) << cut.size_log2, sp.blocks);
        pos += n;
        if (first == last) continue;
        from = sp.first + first * kBlock, to = min(sp.len, sp.first + last * kBlock);
        whole_unit = last - first == sp.blocks;
        if (first == 0 && threadIdx.x == 0) {   // for k_attn_join: segments of the unit
            const int64_t start = rest - off + (int64_t)uni(s_before[b]) * per_seq;
            Parts(a).count[b * (int64_t)per_seq + u] = make_int2(blockIdx.x, (int)((start + length - 1) / cut.share) - blockIdx.x + 1);
        }
        segment = b * (int64_t)per_seq + u + blockIdx.x;
    } else {
        b = blockIdx.x / per_seq, u = blockIdx.x - b * per_seq;
        const int row = uni(row_of(a, b));
        sp = span_of(a, row, uni(len_of(a, row)));
        from = sp.first, to = sp.len;
        pos = end;
    }
    const int hg = u % a.head_groups, j = u / a.head_groups;
    const int heads = min(16, a.group - hg * 16), h0 = j * a.group + hg * 16;

    const int32_t *table = a.table + (int64_t)sp.row * a.width;
    const E *keys = (const E *)a.keys + j * a.c.head_stride, *values = (const E *)a.values + j * a.c.head_stride;
    St st;
    f32x4 acc[NV][VW];
#pragma unroll
    for (int h = 0; h < NV; ++h)
#pragma unroll
        for (int i = 0; i < VW; ++i) acc[h][i] = (f32x4){0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    const float scale = a.scale * kLog2e;

    for (int base = from; base < to; base += kTile) {
        const int n = min(kTile, to - base), padded = (n + TOK - 1) / TOK * TOK;
        if (base > from) __syncthreads();   // places of the tile before are no longer read
        for (int t = threadIdx.x; t < padded; t += 64 * kWaves) {
            int64_t at = -1;
            if (t < n) {
                uint32_t slot;
                const int page = page_of(a.c, table, (uint32_t)(base + t), &slot);
                if (page >= 0) at = page * a.c.page_stride + slot * a.c.slot_stride;
            }
            place[t] = at;
        }
        if (base == from) {   // queries come while the places do; 0 past the heads and past head_dim
            const E *q = (const E *)a.q + b * a.qs.seq + h0 * a.qs.head;
            for (int i = threadIdx.x; i < 16 * DP; i += 64 * kWaves) {
                const int h = i / DP, d = i % DP;
                s_q[h][d] = h < heads && d < D ? q[h * a.qs.head + d * a.qs.dim] : (E)0;
            }
        }
        __syncthreads();
        if (base == from) st.load_q(s_q[r], quad);
        // A step's keys are asked for once the step before has used its own, and likewise its values, so
        // that one of the two is always on its way.  `dead`: the lane's tokens that hold nothing.
        uint32_t dead;
        auto load_k = [&](int s0) __attribute__((always_inline)) {
            int64_t ko[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) ko[t] = place[s0 + 16 * t + r];
            st.template load_k<FULL, ONCE>(keys, ko, quad, D);
            asm volatile("" ::: "memory");   // the loads stay ahead of their use
        };
        auto load_v = [&](int s0) __attribute__((always_inline)) {
            int64_t vo[TT];
            dead = 0;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    vo[4 * t + i] = place[s0 + 16 * t + 4 * quad + i];
                    dead |= (vo[4 * t + i] < 0 ? 1u : 0u) << (4 * t + i);
                }
            st.template load_v<FULL, ONCE>(values, vo, r, D);
            asm volatile("" ::: "memory");
        };
        float s[TT];
        auto softmax = [&]() __attribute__((always_inline)) {
            const bool whole = !__any(dead != 0);
            float top = m;
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                s[i] *= scale;
                if (!whole && (dead >> i & 1)) s[i] = -INFINITY;
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
            if (!whole) st.clear_v(dead);
            if (__any(keep != 1.f))
#pragma unroll
                for (int h = 0; h < NV; ++h)
#pragma unroll
                    for (int i = 0; i < VW; ++i) acc[h][i] *= keep;
            st.outputs(s, acc);
        };
        int s0 = wave * TOK;
        if (s0 < padded) {
            load_k(s0);
            load_v(s0);
            for (;;) {
                st.template scores<FULL>(s, D);
                const int next = s0 + kWaves * TOK;
                if (next >= padded) break;
                load_k(next);
                softmax();
                load_v(next);
                s0 = next;
            }
            softmax();
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
        if (whole_unit) {
            E *y = (E *)a.y + b * a.ys.seq + (h0 + h) * a.ys.head + d * a.ys.dim;
            *y = from_f32<E>(sum == 0.f ? 0.f : o / sum);
            if (d == 0 && a.lse) a.lse[bh] = (ref + log2f(sum)) * kLn2;
        } else {
            const Parts parts(a);
            const int64_t at = parts.at(segment, h);
            parts.o[at * D + d] = o;
            if (d == 0) parts.m[at] = mm, parts.l[at] = sum;
        }
    }
    if (SHARED) __syncthreads();   // the next segment writes these arrays
    }
}

// Joins the segments of a query head: 4 LANES dimensions and 256 / LANES segments at a time, four
// dimensions a thread.  Bound by latency: what a thread's first 8 segments hold is on its way before
// their weights are known (1024 heads of 2 or 3 segments 5.2 us, 6.1 one after the other).
template <typename E, int LANES>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
    constexpr int kAhead = 8, GROUPS = 256 / LANES;
    __shared__ float s_m[kMostShares + 2], s_top[4], s_sum[4];
    __shared__ f32x4 s_o[GROUPS][LANES];
    const int h = blockIdx.x % a.heads, b = blockIdx.x / a.heads, t = threadIdx.x, D = a.c.head_dim;
    const int u = h / a.group * a.head_groups + h % a.group / 16;
    const int64_t unit = (int64_t)b * (a.c.kv_heads * a.head_groups) + u;
    const Parts parts(a);
    const int2 count = parts.count[unit];
    const int n = count.y;
    if (n == 1) return;
    const int64_t seg = unit + count.x;   // the first of n in a row
    const int hh = h % a.group % 16, g = t / LANES, from = blockIdx.y * (4 * LANES), d = from + t % LANES * 4;
    auto finite = [](float top) { return top == -INFINITY ? 0.f : top; };   // what is taken off: -Inf - -Inf is none
    auto out = [&](int p) { return *(const f32x4 *)(parts.o + parts.at(seg + min(p, n - 1), hh) * D + min(d, D - 4)); };
    f32x4 ahead[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i] = out(g + GROUPS * i);
    // of a wave's segments, then of all: maximum, and sum relative to it
    float top = -INFINITY, sum = 0.f;
    for (int p = t; p < n; p += 256) {
        const int64_t at = parts.at(seg + p, hh);
        const float m = parts.m[at], l = parts.l[at], to = fmaxf(top, m), ref = finite(to);
        s_m[p] = m;
        sum = sum * __builtin_amdgcn_exp2f(top - ref) + l * __builtin_amdgcn_exp2f(m - ref);
        top = to;
    }
    float all = top;
    for (int i = 1; i < 64; i *= 2) all = fmaxf(all, __shfl_xor(all, i));
    sum *= __builtin_amdgcn_exp2f(top - finite(all));
    for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
    if (t % 64 == 0) s_top[t / 64] = all, s_sum[t / 64] = sum;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    const float ref = finite(top);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += s_sum[w] * __builtin_amdgcn_exp2f(s_top[w] - ref);
    f32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (g + GROUPS * i < n) v += ahead[i] * __builtin_amdgcn_exp2f(s_m[g + GROUPS * i] - ref);
#pragma unroll 8
    for (int p = g + GROUPS * kAhead; p < n; p += GROUPS) v += out(p) * __builtin_amdgcn_exp2f(s_m[p] - ref);
    s_o[g][t % LANES] = v;
    __syncthreads();
    const int dim = from + t;
    if (t >= 4 * LANES || dim >= D) return;
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) o += ((const float *)s_o[i])[t];
    E *y = (E *)a.y + b * a.ys.seq + h * a.ys.head + dim * a.ys.dim;
    *y = from_f32<E>(sum == 0.f ? 0.f : o / sum);
    if (dim == 0 && a.lse) a.lse[(int64_t)b * a.heads + h] = (ref + log2f(sum)) * kLn2;
}

// Workgroups of a call that is cut into shares: as many as the card holds.
constexpr int shares_of(int dp) { return dp == 256 ? 256 : 512; }
int units_of(const CacheArgs &c, int batch, int heads) {
    return batch * c.kv_heads * ((heads / c.kv_heads + 15) / 16);
}
// Whether the work is cut into shares: for up to kMostSeqs sequences (more fill the card uncut) that may
// be of many steps of a workgroup.  Cutting costs a scan of the lengths and a second kernel, 4 to 10 us,
// and the host 3 us more for a call.  Units that fill the card are worth more steps: 256 of up to 16
// steps take 42 us uncut and 41 cut, 64 sequences of up to 600 tokens 24 and 34; up to 20 steps of 64
// dimensions 48.4 and 46.9.  A few: 8 units of 8 steps 17.1 uncut and 14.3 cut, but in calls by
// themselves 17.3 and 19.5 (64 units of up to 7 steps 17.8 and 19.2); 8 units of 12 steps 22 and 14.5.
// Lengths are on the device, so that the rule goes by the table's width: short sequences in wide tables
// are cut too (1 of 77 tokens 6.9 us in a table as long, 10.6 in one for 8192).
constexpr int kFew = 8, kMany = 16;
// What pays, of sequences of up to `tokens` tokens: never for fewer tokens where not for more.
bool worth_cutting(const CacheArgs &c, int batch, int heads, int64_t tokens) {
    const int64_t steps = tokens / (c.dtype == BSP_F32 ? 64 : 128);
    return batch <= kMostSeqs && steps > (units_of(c, batch, heads) < 256 ? kFew : kMany);
}
// And 32-bit numbers count the blocks of all sequences.  A window may bring them within these again: the
// workspace goes by what may be worth cutting alone.
bool shared(const CacheArgs &c, int batch, int heads, int64_t tokens) {
    return worth_cutting(c, batch, heads, tokens) && batch * (tokens / kBlock + 1 + kCost) <= INT32_MAX;
}

template <typename E, int DP, bool FULL, bool ONCE>
hipError_t run(AttnArgs a, bool split, hipStream_t st) {
    const int units = units_of(a.c, a.batch, a.heads);
    if (!split) {
        k_attn<E, DP, FULL, false, ONCE><<<units, 64 * kWaves, 0, st>>>(a);
        return hipGetLastError();
    }
    a.shares = shares_of(DP);
    k_attn<E, DP, FULL, true, ONCE><<<a.shares, 64 * kWaves, 0, st>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int heads = a.batch * a.heads;
    if (heads < 256)   // few heads: more workgroups for each
        k_attn_join<E, 8><<<dim3(heads, (a.c.head_dim + 31) / 32), 256, 0, st>>>(a);
    else
        k_attn_join<E, 32><<<dim3(heads, (a.c.head_dim + 127) / 128), 256, 0, st>>>(a);
    return hipGetLastError();
}

// Keys and values that are read once (one head group) go past the caches where they could not stay in
// them from one call to the next, half of the last-level one being the bound: 131072 tokens of 8 key
// heads, 537 MB, take 94.6 us past them and 107 through them, 64 sequences of up to 6000 tokens 94 and
// 104; 64 sequences of up to 600 tokens, 41 MB that are still there, 27.4 and 23.5.  How much of a cache
// is in use only the device knows: the rule goes by its pages, and a large one with few tokens in it
// takes the slower side (those 27.4).
template <typename E, int DP, bool FULL>
hipError_t run(const AttnArgs &a, bool split, hipStream_t st) {
    const bool once = a.head_groups == 1 && past_caches(a.c);
    return once ? run<E, DP, FULL, true>(a, split, st) : run<E, DP, FULL, false>(a, split, st);
}

template <typename E>
hipError_t run(const AttnArgs &a, bool split, hipStream_t st) {
    const int D = a.c.head_dim;
    if (D <= 64) return D == 64 ? run<E, 64, true>(a, split, st) : run<E, 64, false>(a, split, st);
    if (D <= 128) return D == 128 ? run<E, 128, true>(a, split, st) : run<E, 128, false>(a, split, st);
    return D == 256 ? run<E, 256, true>(a, split, st) : run<E, 256, false>(a, split, st);
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

// First share and number of segments of every unit; maximum, sum and head_dim outputs of every
// segment, at most shares + units, for each head of a group.  Enough for every window.
int64_t attention_workspace(const CacheArgs &c, int batch, int heads, int width) {
    if (!worth_cutting(c, batch, heads, (int64_t)width * c.page_size)) return 0;
    const int64_t units = units_of(c, batch, heads), segments = kMostShares + units;
    return units * 8 + segments * std::min(16, heads / c.kv_heads) * (c.head_dim + 2) * 4;
}

hipError_t launch_attention(AttnArgs a, hipStream_t st) {
    int64_t tokens = (int64_t)a.width * a.c.page_size;
    if (a.window) tokens = std::min<int64_t>(tokens, a.window);
    a.head_groups = (a.group + 15) / 16;
    a.shares = 0;
    const bool split = shared(a.c, a.batch, a.heads, tokens);
    return a.c.dtype == BSP_F32 ? run<float>(a, split, st) : run<uint16_t>(a, split, st);
}

}  // namespace bsp
