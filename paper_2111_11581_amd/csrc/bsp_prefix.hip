// Attention of one new token of each sequence over a paged cache, where groups of sequences share the
// pages of their first tokens.
//
// What a group shares is one matrix of keys and values for the queries of all its members: of a key
// head, members times the query heads that share it are the columns of the products, 64 at a time (32
// for more than 128 dimensions), all of which a wave holds in registers; it reads each key and value once
// for them, straight from memory into the operands as k_attn does.  What a member has of its own is a
// group of one.  Both are cut into shares for the workgroups, and k_prefix_join joins the parts of
// every query head by their maxima.
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_attn.h"

namespace bsp {

namespace {

constexpr int kShares = 256;            // workgroups that the work is cut for: one a CU, for its registers
constexpr int kMost = kMostPrefixSeqs;
constexpr int columns_of(int dp) { return dp == 256 ? 32 : 64; }
int dims_of(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// Work is counted in thirds of the time that reading 32 tokens from memory takes a CU; beginning and
// ending a segment is worth eight of these.
constexpr int kOwn = 3, kCost = 24, kMinShare = kCost + 24;

// The most units that there may be: of what groups share (a group's columns of a key head), and of what
// sequences have of their own (up to 16 query heads of a key head).
struct Units {
    int64_t shared, own;
};
Units units_of(const CacheArgs &c, int batch, int heads, int groups) {
    const int group = heads / c.kv_heads;
    Units u;
    u.shared = groups ? ((int64_t)batch * group / columns_of(dims_of(c.head_dim)) + groups) * c.kv_heads : 0;
    u.own = (int64_t)batch * c.kv_heads * ((group + 15) / 16);
    return u;
}

// The workspace: outputs, maxima and sums of the columns of segments (share g and unit u of either kind
// meet in at most one, g + u of the kind's own); first share and number of segments of every unit; of
// every sequence its group's first unit, that unit's columns and its own place among them.
struct Parts {
    float *o, *m, *l;
    int columns;
    __device__ __forceinline__ int64_t at(int64_t segment, int column) const { return segment * columns + column; }
};
struct Space {
    Parts shared, own;
    int2 *shared_count, *own_count;
    int4 *member;
    int64_t bytes;
};
__host__ __device__ inline Space space_of(void *workspace, const Units &u, int batch, int columns, int own_columns, int head_dim) {
    Space s;
    char *at = (char *)workspace;
    auto take = [&](int64_t bytes) {
        char *here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    auto parts = [&](int64_t units, int cols) {
        const int64_t n = units ? (kShares + units) * cols : 0;
        Parts p;
        p.columns = cols, p.o = (float *)take(n * head_dim * 4), p.m = (float *)take(n * 4), p.l = (float *)take(n * 4);
        return p;
    };
    s.shared = parts(u.shared, columns), s.own = parts(u.own, own_columns);
    s.shared_count = (int2 *)take(u.shared * 8), s.own_count = (int2 *)take(u.own * 8);
    s.member = (int4 *)take((int64_t)batch * 16);
    s.bytes = at - (char *)workspace;
    return s;
}

// The work in a row: what groups share, then what sequences have of their own; an item is some units of
// one length.  Every workgroup works it out for itself.
struct Item {
    int units, blocks, weight;
    __device__ __forceinline__ int length() const { return blocks ? blocks * weight + kCost : 0; }
};
struct Plan {
    int len[kMost];                           // of sequences
    int16_t group[kMost];                     // or -1
    int lo[kMost + 1];                        // group g: entries lo[g] to lo[g + 1]
    int from[kMost], to[kMost];               // tokens that any of its members attends to
    int64_t before[2 * kMost + 1];            // length of all items before
    int unit[kMost];                          // number of a group's first unit
    int64_t wave[kWaves];

    __device__ __forceinline__ int tokens_from(const AttnArgs &a, int b) const {
        return a.window && len[b] > a.window ? len[b] - a.window : 0;
    }
    __device__ __forceinline__ int shared_of(const PrefixArgs &p, int g) const { return g < 0 ? 0 : max(0, p.shared[g]); }
    __device__ __forceinline__ Item item(const PrefixArgs &p, int columns_of_unit, int i) const {
        const AttnArgs &a = p.a;
        Item it;
        if (i < p.groups) {
            const int columns = (lo[i + 1] - lo[i]) * a.group, n = (columns + columns_of_unit - 1) / columns_of_unit;
            it.units = n * a.c.kv_heads, it.blocks = (max(0, to[i] - from[i]) + kBlock - 1) / kBlock;
            it.weight = n >= 3 ? 1 : 4 - n;   // more workgroups that read the same
        } else {
            const int b = i - p.groups, first = max(tokens_from(a, b), shared_of(p, group[b]));
            it.units = a.c.kv_heads * a.head_groups, it.weight = kOwn;
            it.blocks = (int)(((int64_t)max(0, len[b] - first) + kBlock - 1) / kBlock);
        }
        return it;
    }
};

// Inclusive scan over the workgroup of one value a thread; *all: of all of them.
template <typename T, typename F> __device__ __forceinline__ T scan(T v, T *s_wave, T *all, F join) {
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    for (int d = 1; d < 64; d *= 2) {
        const T o = __shfl_up(v, d);
        if (lane >= d) v = join(v, o);
    }
    __syncthreads();
    if (lane == 63) s_wave[w] = v;
    __syncthreads();
    T before = s_wave[0];
    *all = before;
    T mine = v;
#pragma unroll
    for (int i = 1; i <= kWaves; ++i) {
        if (i == w) mine = join(v, before);
        if (i < kWaves) before = join(before, s_wave[i]);
    }
    *all = before;
    return mine;
}

template <int COLUMNS> __device__ __forceinline__ int64_t make_plan(const PrefixArgs &p, Plan &s) {
    const AttnArgs &a = p.a;
    const int t = threadIdx.x, G = p.groups;
    for (int b = t; b < a.batch; b += 64 * kWaves) s.len[b] = len_of(a, row_of(a, b));
    if (G) {
        // bounds in order and within the batch, whatever starts holds
        const int per = (G + 64 * kWaves) / (64 * kWaves);
        int64_t top = 0, all;
        for (int i = t * per; i < min(G + 1, (t + 1) * per); ++i) top = max(top, (int64_t)min(max(p.starts[i], 0), a.batch));
        top = scan(top, s.wave, &all, [](int64_t x, int64_t y) { return max(x, y); });
        int64_t upto = __shfl_up(top, 1);
        if (t % 64 == 0) {
            upto = 0;
            for (int w = 0; w < t / 64; ++w) upto = max(upto, s.wave[w]);
        }
        for (int i = t * per; i < min(G + 1, (t + 1) * per); ++i) {
            upto = max(upto, (int64_t)min(max(p.starts[i], 0), a.batch));
            s.lo[i] = (int)upto;
        }
        for (int g = t; g < G; g += 64 * kWaves) s.from[g] = INT32_MAX, s.to[g] = 0;
        __syncthreads();
        for (int b = t; b < a.batch; b += 64 * kWaves) {
            int lo = 0, hi = G;   // the last group that begins at or before b
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (s.lo[mid] <= b) lo = mid; else hi = mid;
            }
            const int g = b >= s.lo[lo] && b < s.lo[lo + 1] ? lo : -1;
            s.group[b] = (int16_t)g;
            const int first = s.tokens_from(a, b), last = min(s.len[b], s.shared_of(p, g));
            if (g >= 0 && first < last) atomicMin(&s.from[g], first), atomicMax(&s.to[g], last);
        }
    } else {
        for (int b = t; b < a.batch; b += 64 * kWaves) s.group[b] = -1;
    }
    __syncthreads();
    const int items = G + a.batch, per = (items + 64 * kWaves - 1) / (64 * kWaves);
    int64_t sum = 0, total, units = 0, all_units;
    for (int i = t * per; i < min(items, (t + 1) * per); ++i) {
        const Item it = s.item(p, COLUMNS, i);
        sum += (int64_t)it.units * it.length(), units += it.units;
    }
    auto add = [](int64_t x, int64_t y) { return x + y; };
    int64_t upto = scan(sum, s.wave, &total, add) - sum;
    units = scan(units, s.wave, &all_units, add) - units;
    for (int i = t * per; i < min(items, (t + 1) * per); ++i) {
        const Item it = s.item(p, COLUMNS, i);
        s.before[i] = upto;
        if (i < G) s.unit[i] = (int)units;
        upto += (int64_t)it.units * it.length(), units += it.units;
    }
    if (t == 0) s.before[items] = total;
    __syncthreads();
    return total;
}

// Tokens from .. to of a row of the table, for `columns` columns from column c0 on: query head c % group
// of key head j and sequence first + c / group.
struct Segment {
    int row, j, first, c0, columns, from, to;
    Parts parts;
    int64_t number;
};

template <typename E, int DP> struct Shared {
    static constexpr int COLUMNS = columns_of(DP), ROW = DP + 4;
    Plan plan;
    int64_t place[kTile];
    float m[kWaves][16], l[kWaves][16];
    __attribute__((aligned(16))) float o[2][16][ROW];
    __attribute__((aligned(16))) E q[COLUMNS][DP + 16 / sizeof(E)];
};

// A segment by a workgroup, its waves in turn for the tokens; N: columns in sixteens.  A column's reference
// of the softmax is not its maximum but within 2^6 of it, or above: it moves only where some score passes
// it by so much, which costs a vote a step instead of two exchanges and a product for every output.
template <typename E, int DP, bool FULL, int N>
__device__ __forceinline__ void run_segment(const PrefixArgs &p, Shared<E, DP> &sh, const Segment &g) {
    typedef Step<E, DP> St;
    constexpr int TOK = St::TOK, TT = TOK / 4, NT = TOK / 16, VW = St::VW, NV = St::NV;
    constexpr float kPast = 6.f;
    const AttnArgs &a = p.a;
    const int D = a.c.head_dim, wave = uni(threadIdx.x / 64);
    int lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));   // what goes by the lane is worked out again for each segment, not held in registers
    const int r = lane % 16, quad = lane / 16;
    const int32_t *table = a.table + (int64_t)g.row * a.width;
    const bool in = (unsigned)g.row < (unsigned)a.seqs;
    const E *keys = (const E *)a.keys + g.j * a.c.head_stride, *values = (const E *)a.values + g.j * a.c.head_stride;

    St st;
    typename St::Quad q[N][St::NK];
    f32x4 acc[N][NV][VW];
    float m[N], l[N];
    int begin[N], end[N];   // tokens that a lane's columns attend to
    int all_from = 0, all_to = INT32_MAX;   // those that every column does
#pragma unroll
    for (int n = 0; n < N; ++n) {
        m[n] = -INFINITY, l[n] = 0.f;
        begin[n] = 0, end[n] = INT32_MAX;
        if (n * 16 + r < g.columns) {
            const int b = g.first + (g.c0 + n * 16 + r) / a.group;
            begin[n] = sh.plan.tokens_from(a, b), end[n] = sh.plan.len[b];
        }
        all_from = max(all_from, begin[n]), all_to = min(all_to, end[n]);
#pragma unroll
        for (int h = 0; h < NV; ++h)
#pragma unroll
            for (int i = 0; i < VW; ++i) acc[n][h][i] = (f32x4){0, 0, 0, 0};
    }
    for (int d = 1; d < 16; d *= 2) all_from = max(all_from, __shfl_xor(all_from, d)), all_to = min(all_to, __shfl_xor(all_to, d));
    all_from = uni(all_from), all_to = uni(all_to);
    // scores in powers of two; queries change their sign with the scale's, so that a larger product is a larger score
    const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * kLog2e;
    const float by = a.scale == 0.f ? 0.f : a.scale < 0.f ? -1.f : 1.f;

    for (int base = g.from; base < g.to; base += kTile) {
        const int n = min(kTile, g.to - base), padded = (n + TOK - 1) / TOK * TOK;
        __syncthreads();   // places and queries of the tile before are no longer read
        for (int t = threadIdx.x; t < padded; t += 64 * kWaves) {
            int64_t at = -1;
            if (in && t < n) {
                uint32_t slot;
                const int page = page_of(a.c, table, (uint32_t)(base + t), &slot);
                if (page >= 0) at = page * a.c.page_stride + slot * a.c.slot_stride;
            }
            sh.place[t] = at;
        }
        if (base == g.from) {   // queries come while the places do, along the way they lie; 0 past columns and head_dim
            const bool by_column = a.qs.dim != 1;
            for (int i = threadIdx.x; i < 16 * N * DP; i += 64 * kWaves) {
                const int c = by_column ? i % (16 * N) : i / DP, d = by_column ? i / (16 * N) : i % DP, at = g.c0 + c;
                E v = (E)0;
                if (c < g.columns && d < D) {
                    const int k = at / a.group;
                    v = ((const E *)a.q)[(g.first + k) * a.qs.seq + (g.j * a.group + at - k * a.group) * a.qs.head + d * a.qs.dim];
                    if (by != 1.f) v = from_f32<E>(to_f32(v) * by);
                }
                sh.q[c][d] = v;
            }
        }
        __syncthreads();
        if (base == g.from)
#pragma unroll
            for (int n = 0; n < N; ++n) St::load_q(q[n], sh.q[n * 16 + r], quad);
        uint32_t dead;   // the lane's tokens that hold nothing
        auto load_k = [&](int s0) __attribute__((always_inline)) {
            int64_t ko[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) ko[t] = sh.place[s0 + 16 * t + r];
            st.template load_k<FULL, false>(keys, ko, quad, D);
            asm volatile("" ::: "memory");   // the loads stay ahead of their use
        };
        auto load_v = [&](int s0) __attribute__((always_inline)) {
            int64_t vo[TT];
            dead = 0;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    vo[4 * t + i] = sh.place[s0 + 16 * t + 4 * quad + i];
                    dead |= (vo[4 * t + i] < 0 ? 1u : 0u) << (4 * t + i);
                }
            st.template load_v<FULL, false>(values, vo, r, D);
            asm volatile("" ::: "memory");
        };
        float s[N][TT];
        auto softmax = [&](int s0) __attribute__((always_inline)) {
            const int t0 = base + s0;
            const bool whole = t0 >= all_from && t0 + TOK <= all_to && !__any(dead != 0);
            uint32_t out[N];   // a lane's tokens that its columns do not attend to
            if (!whole) {
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    out[n] = dead;
#pragma unroll
                    for (int i = 0; i < TT; ++i) {
                        const int t = t0 + 16 * (i / 4) + 4 * quad + i % 4;
                        if (t < begin[n] || t >= end[n]) out[n] |= 1u << i;
                        if (out[n] >> i & 1) s[n][i] = -INFINITY;
                    }
                }
                st.clear_v(dead);
            }
            float top[N];
            bool past = false;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                top[n] = s[n][0];
#pragma unroll
                for (int i = 1; i < TT; ++i) top[n] = fmaxf(top[n], s[n][i]);
                top[n] *= scale;
                past |= top[n] > m[n] + kPast;
            }
            if (__any(past))
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float to = fmaxf(top[n], __shfl_xor(top[n], 16));
                    to = fmaxf(m[n], fmaxf(to, __shfl_xor(to, 32)));
                    const float keep = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - to);
                    m[n] = to, l[n] *= keep;
#pragma unroll
                    for (int h = 0; h < NV; ++h)
#pragma unroll
                        for (int i = 0; i < VW; ++i) acc[n][h][i] *= keep;
                }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const float ref = m[n] == -INFINITY ? 0.f : m[n];
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < TT; ++i) {
                    s[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], scale, -ref));
                    if (!whole && (out[n] >> i & 1)) s[n][i] = 0.f;
                    sum += s[n][i];
                }
                l[n] += sum;
            }
            st.template outputs<N>(s, acc);
        };
        int s0 = wave * TOK;
        if (s0 < padded) {
            load_k(s0);
            load_v(s0);
            for (;;) {
#pragma unroll
                for (int n = 0; n < N; ++n) st.template scores<FULL>(q[n], s[n], D);
                const int next = s0 + kWaves * TOK;
                if (next >= padded) break;
                load_k(next);
                softmax(s0);
                load_v(next);
                s0 = next;
            }
            softmax(s0);
        }
    }

    // join the waves, sixteen columns at a time: all on the common reference, then 2 and 3 onto 0 and 1
#pragma unroll
    for (int n = 0; n < N; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (n) __syncthreads();   // the sixteen before have been read
        if (quad == 0) sh.m[wave][r] = m[n], sh.l[wave][r] = l[n];
        __syncthreads();
        float top = sh.m[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh.m[w][r]);
        const float f = __builtin_amdgcn_exp2f(m[n] - (top == -INFINITY ? 0.f : top));
        for (int turn = 0; turn < 2; ++turn) {
            if (wave / 2 == 1 - turn)
#pragma unroll
                for (int h = 0; h < NV; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int v = 0; v < VW; v += 4) {
                            f32x4 *o = (f32x4 *)&sh.o[wave % 2][r][h * 16 * VW + (quad * 4 + i) * VW + v];
                            f32x4 x = {acc[n][h][v][i], acc[n][h][v + 1][i], acc[n][h][v + 2][i], acc[n][h][v + 3][i]};
                            x *= f;
                            *o = turn ? *o + x : x;
                        }
            __syncthreads();
        }
        const int columns = min(16, g.columns - n * 16);
        for (int i = threadIdx.x; i < columns * DP; i += 64 * kWaves) {
            const int c = i / DP, d = i % DP;
            if (d >= D) continue;
            const int64_t at = g.parts.at(g.number, n * 16 + c);
            g.parts.o[at * D + d] = sh.o[0][c][d] + sh.o[1][c][d];
            if (d == 0) {
                float mm = sh.m[0][c], sum = 0.f;
#pragma unroll
                for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, sh.m[w][c]);
                const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += sh.l[w][c] * __builtin_amdgcn_exp2f(sh.m[w][c] - ref);
                g.parts.m[at] = mm, g.parts.l[at] = sum;
            }
        }
    }
    __syncthreads();   // the next segment writes these arrays
}

template <typename E, int DP, bool FULL>
__global__ __launch_bounds__(64 * kWaves, 1) void k_prefix(PrefixArgs p, Units units) {
    constexpr int COLUMNS = columns_of(DP);
    __shared__ Shared<E, DP> sh;
    const AttnArgs &a = p.a;
    const int G = p.groups, items = G + a.batch;
    // consecutive shares on one XCD, whose L2 then holds what several of them read
    const int share_number = blockIdx.x % 8 * (kShares / 8) + blockIdx.x / 8;
    const Space space = space_of(a.workspace, units, a.batch, COLUMNS, min(16, a.group), a.c.head_dim);
    const int64_t total = make_plan<COLUMNS>(p, sh.plan);
    const int64_t share = max((int64_t)kMinShare, (total + kShares - 1) / kShares);

    // for k_prefix_join: where a member's columns are, and units without tokens
    int64_t pos = share_number * share;
    const int64_t end = min(pos + share, total);
    for (int i = share_number; i < items; i += kShares) {
        const Item it = sh.plan.item(p, COLUMNS, i);
        if (i >= G) {
            const int b = i - G, g = sh.plan.group[b];
            if (threadIdx.x == 0) {
                space.member[b] = g < 0 ? make_int4(-1, 0, 0, 0) :
                    make_int4(sh.plan.unit[g], sh.plan.item(p, COLUMNS, g).units / a.c.kv_heads, b - sh.plan.lo[g], 0);
            }
        }
        if (it.blocks) continue;
        int2 *count = i < G ? space.shared_count + sh.plan.unit[i] : space.own_count + (int64_t)(i - G) * it.units;
        for (int u = threadIdx.x; u < it.units; u += 64 * kWaves) count[u] = make_int2(0, 0);
    }

    while (pos < end) {
        int lo = 0, hi = items;   // the last item that begins at or before pos, which has length
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (sh.plan.before[mid] <= pos) lo = mid; else hi = mid;
        }
        const int i = uni(lo);
        const Item it = sh.plan.item(p, COLUMNS, i);
        const int length = uni(it.length()), weight = uni(it.weight);
        const int64_t rest = pos - sh.plan.before[i];
        const int u = uni((int)(rest / length)), off = uni((int)(rest - (int64_t)u * length));
        const int n = uni((int)min(end - pos, (int64_t)(length - off)));
        const int first = max(0, off - kCost) / weight, last = max(0, off + n - kCost) / weight;   // blocks of the segment
        const int64_t start = pos - off;
        pos += n;
        if (first == last) continue;
        Segment g;
        int64_t unit;
        int2 *count;
        int whole_from, whole_to;
        if (i < G) {
            const int blocks = uni(it.units) / a.c.kv_heads, all = (uni(sh.plan.lo[i + 1]) - uni(sh.plan.lo[i])) * a.group;
            g.first = uni(sh.plan.lo[i]), g.j = u / blocks, g.c0 = (u - g.j * blocks) * COLUMNS;
            g.columns = min(COLUMNS, all - g.c0);
            g.row = uni(p.prefix_rows ? p.prefix_rows[i] : row_of(a, g.first));
            whole_from = uni(sh.plan.from[i]), whole_to = uni(sh.plan.to[i]);
            unit = uni(sh.plan.unit[i]) + u, count = space.shared_count + unit, g.parts = space.shared;
        } else {
            const int b = i - G;
            g.first = b, g.j = u / a.head_groups, g.c0 = (u - g.j * a.head_groups) * 16;
            g.columns = min(16, a.group - g.c0);
            g.row = uni(row_of(a, b));
            whole_from = uni(max(sh.plan.tokens_from(a, b), sh.plan.shared_of(p, sh.plan.group[b]))), whole_to = uni(sh.plan.len[b]);
            unit = (int64_t)b * it.units + u, count = space.own_count + unit, g.parts = space.own;
        }
        g.from = whole_from + first * kBlock, g.to = min(whole_to, whole_from + last * kBlock);
        g.number = share_number + unit;
        if (first == 0 && threadIdx.x == 0)
            *count = make_int2(share_number, (int)((start + length - 1) / share) - share_number + 1);
        if (g.columns <= 16)
            run_segment<E, DP, FULL, 1>(p, sh, g);
        else if (g.columns <= 32 || COLUMNS == 32)
            run_segment<E, DP, FULL, 2>(p, sh, g);
        else if constexpr (COLUMNS == 64)
            run_segment<E, DP, FULL, 4>(p, sh, g);
    }
}

// Joins the segments of a query head, those of its group and its own: 4 dimensions a thread, eight segments
// at a time.
template <typename E>
__global__ __launch_bounds__(256) void k_prefix_join(PrefixArgs p, Units units, int columns) {
    constexpr int LANES = 32, GROUPS = 256 / LANES;
    __shared__ float s_m[2 * kShares + 2], s_top[4], s_sum[4];
    __shared__ f32x4 s_o[GROUPS][LANES];
    const AttnArgs &a = p.a;
    const int h = blockIdx.x % a.heads, b = blockIdx.x / a.heads, t = threadIdx.x, D = a.c.head_dim;
    const int j = h / a.group, hh = h - j * a.group, own_columns = min(16, a.group);
    const Space space = space_of(a.workspace, units, a.batch, columns, own_columns, D);
    const int64_t own_unit = ((int64_t)b * a.c.kv_heads + j) * a.head_groups + hh / 16;
    const int4 member = space.member[b];
    const int2 own = space.own_count[own_unit];
    int2 shared = make_int2(0, 0);
    int64_t shared_unit = 0;
    int column = 0;
    if (member.x >= 0) {
        column = member.z * a.group + hh;
        shared_unit = member.x + (int64_t)j * member.y + column / columns, column %= columns;
        shared = space.shared_count[shared_unit];
    }
    const int n = shared.y + own.y;
    auto at = [&](int k, const Parts **parts) {
        if (k < shared.y) {
            *parts = &space.shared;
            return space.shared.at(shared_unit + shared.x + k, column);
        }
        *parts = &space.own;
        return space.own.at(own_unit + own.x + k - shared.y, hh % 16);
    };
    auto finite = [](float top) { return top == -INFINITY ? 0.f : top; };   // what is taken off: -Inf - -Inf is none
    float top = -INFINITY, sum = 0.f;
    for (int k = t; k < n; k += 256) {
        const Parts *parts;
        const int64_t i = at(k, &parts);
        const float m = parts->m[i], l = parts->l[i], to = fmaxf(top, m), ref = finite(to);
        s_m[k] = m;
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
    const int from = blockIdx.y * (4 * LANES), d = from + t % LANES * 4;
    f32x4 v = {0, 0, 0, 0};
    for (int k = t / LANES; k < n; k += GROUPS) {
        const Parts *parts;
        const int64_t i = at(k, &parts);
        v += *(const f32x4 *)(parts->o + i * D + min(d, D - 4)) * __builtin_amdgcn_exp2f(s_m[k] - ref);
    }
    s_o[t / LANES][t % LANES] = v;
    __syncthreads();
    const int dim = from + t;
    if (t >= 4 * LANES || dim >= D) return;
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) o += ((const float *)s_o[i])[t];
    ((E *)a.y)[b * a.ys.seq + h * a.ys.head + dim * a.ys.dim] = from_f32<E>(sum == 0.f ? 0.f : o / sum);
    if (dim == 0 && a.lse) a.lse[(int64_t)b * a.heads + h] = (ref + log2f(sum)) * kLn2;
}

template <typename E, int DP, bool FULL> hipError_t run(const PrefixArgs &p, const Units &units, hipStream_t st) {
    k_prefix<E, DP, FULL><<<kShares, 64 * kWaves, 0, st>>>(p, units);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const dim3 grid(p.a.batch * p.a.heads, (p.a.c.head_dim + 127) / 128);
    k_prefix_join<E><<<grid, 256, 0, st>>>(p, units, columns_of(DP));
    return hipGetLastError();
}

template <typename E> hipError_t run(const PrefixArgs &p, const Units &units, hipStream_t st) {
    const int D = p.a.c.head_dim;
    if (D <= 64) return D == 64 ? run<E, 64, true>(p, units, st) : run<E, 64, false>(p, units, st);
    if (D <= 128) return D == 128 ? run<E, 128, true>(p, units, st) : run<E, 128, false>(p, units, st);
    return D == 256 ? run<E, 256, true>(p, units, st) : run<E, 256, false>(p, units, st);
}

}  // namespace

int64_t prefix_workspace(const CacheArgs &c, int batch, int heads, int groups, int) {
    const Units u = units_of(c, batch, heads, groups);
    return space_of(nullptr, u, batch, columns_of(dims_of(c.head_dim)), std::min(16, heads / c.kv_heads), c.head_dim).bytes;
}

hipError_t launch_prefix(const PrefixArgs &args, hipStream_t st) {
    PrefixArgs p = args;
    p.a.head_groups = (p.a.group + 15) / 16, p.a.shares = kShares;
    const Units u = units_of(p.a.c, p.a.batch, p.a.heads, p.groups);
    return p.a.c.dtype == BSP_F32 ? run<float>(p, u, st) : run<uint16_t>(p, u, st);
}

}  // namespace bsp
