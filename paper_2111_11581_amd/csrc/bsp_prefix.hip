// Attention of one new token of each sequence over a paged cache, where groups of sequences share the
// pages of their first tokens.
//
// What a group shares is one matrix of keys and values for the queries of all its members: of a key
// head, members times the query heads that share it are the columns of the products.  What a member
// has of its own is a group of one.
//  * k_prefix_plan cuts both into tasks of about equal cost, by lengths that only the device knows.
//  * k_prefix works on the tasks, of which every workgroup takes the next one when it has done its
//    last.  Up to 32 columns go as in k_attn: keys and values come straight from memory into the
//    operands, the waves take the tokens in turn (columns_narrow).  More, up to 256, share what is
//    staged in LDS, 32 a wave (columns_wide).
//  * k_prefix_join joins the tasks of every query head by their maxima, in the order of their tokens.
// Tables that hold few tokens take one kernel instead (k_prefix_short).
// 32 sequences over 4096 shared tokens (34 MB) take 34 us in a graph: a plan of 8, tasks of 20 and a join of 6, each
// a chain of latencies.  64 over 32768 (69 GFLOP, half as many again for probabilities in two parts) take 149: tasks
// of 138, in which MFMA works 37 % of the time and VALU 47 %.  Without tokens of their own, which are 512 short tasks after
// the shared ones, 16 less, whether they are 1 or 128 for a sequence.
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_attn.h"

namespace bsp {

namespace {

constexpr int kMost = kMostPrefixSeqs;
constexpr int kGrid = 256;              // workgroups: one a CU
constexpr int kStep = 128;              // tokens by which work is cut, and that are staged at a time
constexpr int kRounds = 2;              // tasks a workgroup at most, but for what cannot be cut smaller
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;

// Columns of a task: staged ones only for what fits LDS and registers.
template <typename E, int DP> constexpr int kColumns = sizeof(E) == 2 && DP <= 128 ? 256 : 32;
int dims_of(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
int columns_of(int dtype, int head_dim) { return dtype == BSP_BF16 && head_dim <= 128 ? 256 : 32; }
// Waves of k_prefix: two for a SIMD, or one where a wave's registers ask for it.
template <int DP> constexpr int kTaskWaves = DP == 256 ? 4 : 8;

// ---- the workspace ---------------------------------------------------------------------------------

// Columns c0 .. of key head j, from sequence `first` on, over tokens number from .. to of a list: number i is token
// begin + i, and `skip` more from number `cut` on; those below `shared` are in the pages of row `lead`.  With `units` above 0
// these are so many units of sequence `first` side by side, from number j on, a unit being up to 16 query heads of a key head.
struct Task {
    int j, first, c0, columns, from, to;
    int row, lead, shared, begin, cut, skip;
    int number, units, unused[2];   // number: among all tasks
};
struct Member {
    int task, blocks, pieces, place;   // the group's first task, column blocks, pieces; place in the group
    int own_task, own_pieces, unused[2];
};
struct Head {
    int tasks, shared;        // all, and of those the ones of what groups share, which come first
    int next, bundle;         // the next one to take; log2 of the units in a task of what sequences have of their own
    int zero[4];
};
struct Parts {
    float *o, *m, *l;
    int columns;
    __device__ __forceinline__ int64_t at(int64_t task, int column) const { return task * columns + column; }
};
struct Space {
    Head *head;
    void *q;                  // queries [batch][heads][dims], 0 past head_dim, of the scale's sign
    Member *member;
    Task *task;
    Parts shared, own;
    int64_t bytes;
};
// Of either kind there are as many tasks as units, which nothing cuts, and kRounds * kGrid more at most: a unit's pieces are
// one more than its cost over the cost of all over kRounds * kGrid, rounded down.
struct Sizes {
    int64_t shared_tasks, own_tasks, own_parts, query_bytes;
    int columns, own_columns;
    int bundle_log2;   // units of a sequence's own in a task, at most
};
Sizes sizes_of(const CacheArgs &c, int batch, int heads, int groups) {
    const int64_t group = heads / c.kv_heads;
    Sizes s;
    const int block = columns_of(c.dtype, c.head_dim);
    s.columns = (int)std::min<int64_t>(block, (batch * group + 15) / 16 * 16);
    s.own_columns = (int)std::min<int64_t>(16, group);
    s.query_bytes = (int64_t)batch * heads * dims_of(c.head_dim) * (c.dtype == BSP_F32 ? 4 : 2);
    s.shared_tasks = groups ? (batch * group / block + groups) * c.kv_heads + kRounds * kGrid : 0;
    const int64_t per_seq = c.kv_heads * ((group + 15) / 16);
    s.bundle_log2 = 0;
    while (s.bundle_log2 < (c.head_dim > 128 ? 2 : 3) && 2 << s.bundle_log2 <= per_seq && batch * per_seq >> (s.bundle_log2 + 1) >= kGrid / 4)
        ++s.bundle_log2;
    s.own_tasks = batch * per_seq + kRounds * kGrid;
    s.own_parts = batch * (per_seq + (1 << s.bundle_log2) - 1) + ((int64_t)kRounds * kGrid << s.bundle_log2);
    return s;
}
__host__ __device__ inline Space space_of(void *workspace, const Sizes &z, int batch, int head_dim) {
    Space s;
    char *at = (char *)workspace;
    auto take = [&](int64_t bytes) {
        char *here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    auto parts = [&](int64_t tasks, int columns) {
        Parts p;
        const int64_t n = tasks * columns;
        p.columns = columns, p.o = (float *)take(n * head_dim * 4), p.m = (float *)take(n * 4), p.l = (float *)take(n * 4);
        return p;
    };
    s.head = (Head *)take(sizeof(Head)), s.q = take(z.query_bytes), s.member = (Member *)take((int64_t)batch * sizeof(Member));
    s.task = (Task *)take((kGrid + z.shared_tasks + z.own_tasks) * sizeof(Task));
    s.shared = parts(z.shared_tasks, z.columns), s.own = parts(z.own_parts, z.own_columns);
    s.bytes = at - (char *)workspace;
    return s;
}

// The factor of scores in powers of two, and the sign that queries take instead of it, so that a larger product is a
// larger score; a scale of 0 makes queries of 0.
struct Scale {
    float by, sign;
    __device__ __forceinline__ explicit Scale(float scale)
        : by(scale == 0.f ? 1.f : fabsf(scale) * kLog2e), sign(scale == 0.f ? 0.f : scale < 0.f ? -1.f : 1.f) {}
    template <typename E> __device__ __forceinline__ E of(E v) const { return sign == 1.f ? v : from_f32<E>(to_f32(v) * sign); }
};

// ---- the plan ----------------------------------------------------------------------------------------

// What 128 tokens cost a CU, in units of 1800 cycles: reading keys and values of 128 dimensions from memory takes
// 4 of these for bf16 and 8 for fp32 (less each where several column blocks read the same), the products 1 for
// every 64 columns of bf16 and 5 for 32 of fp32.  A task by itself is worth kTaskCost.
constexpr int kTaskCost = 8, kLeastTask = 16;   // the latter: the least that a task is cut to
__device__ __forceinline__ int cost_of(bool f32, int columns, int blocks) {
    const int read = f32 ? 8 : 4, compute = f32 ? 5 * ((columns + 31) / 32) : (columns + 63) / 64;
    return max((read + blocks - 1) / blocks, compute);
}

// Inclusive scan of one value a thread over the workgroup; 0 adds nothing.
template <typename T, typename F> __device__ __forceinline__ T scan(T v, T *s_wave, F join) {
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    v = wave_scan(v, join);
    __syncthreads();
    if (lane == 63) s_wave[w] = v;
    __syncthreads();
    for (int i = 0; i < w; ++i) v = join(s_wave[i], v);
    return v;
}

// Queries as a task's lanes read them, 16 bytes a thread, along the sequences where these lie side by side.  Staged by each
// task instead, k_prefix takes 39 us for 32 sequences over 4096 tokens, and 31 so.
template <typename E, int DP> __device__ __forceinline__ void lay_queries(const AttnArgs &a, E *to, int64_t i) {
    constexpr int VE = 16 / sizeof(E), N = DP / VE;
    const int rows = a.batch * a.heads;
    if (i >= (int64_t)rows * N) return;
    int b, h, d0;
    if (a.qs.dim == 1) d0 = (int)(i % N) * VE, h = (int)(i / N % a.heads), b = (int)(i / N / a.heads);
    else b = (int)(i % a.batch), d0 = (int)(i / a.batch % N) * VE, h = (int)(i / a.batch / N);
    const E *q = (const E *)a.q + b * a.qs.seq + h * a.qs.head;
    const Scale scale(a.scale);
    __attribute__((aligned(16))) E v[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = q[min(d0 + e, a.c.head_dim - 1) * a.qs.dim];
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = d0 + e < a.c.head_dim ? scale.of(v[e]) : (E)0;
    *(u32x4 *)(to + ((int64_t)b * a.heads + h) * DP + d0) = *(const u32x4 *)v;
}

// Block 0 plans, a thread for a group and for a sequence: as many waves as these need, since each wave makes every
// scan and sum longer, but four at least.  The other blocks lay the queries out meanwhile.  Bound by latency: 8 us for
// 32 sequences.
template <typename E, int DP> __global__ __launch_bounds__(kMost) void k_prefix_plan(PrefixArgs p, Sizes z, int block_columns) {
    if (blockIdx.x > 0) {
        const Space space = space_of(p.a.workspace, z, p.a.batch, p.a.c.head_dim);
        lay_queries<E, DP>(p.a, (E *)space.q, (int64_t)(blockIdx.x - 1) * blockDim.x + threadIdx.x);
        return;
    }
    constexpr int MOST = kMost / 64;
    const int T = blockDim.x, W = T / 64;
    __shared__ int s_lo[kMost + 1], s_from[kMost], s_to[kMost], s_wave[MOST];
    __shared__ int s_task[2 * kMost + 1], s_pieces[2 * kMost], s_steps[2 * kMost];
    __shared__ struct {
        int row, lead, shared, begin, cut, skip, len;
    } s_own[kMost];
    __shared__ int64_t s_sum[MOST][5], s_all;
    const AttnArgs &a = p.a;
    const int t = threadIdx.x, G = p.groups, B = a.batch;
    const Space space = space_of(a.workspace, z, B, a.c.head_dim);
    const bool f32 = a.c.dtype == BSP_F32;
    auto bound = [&](int g) { return min(max(p.starts[g], 0), B); };

    const int row = t < B ? row_of(a, t) : -1, len = t < B ? len_of(a, row) : 0;
    const int begin = a.window && len > a.window ? len - a.window : 0;
    int group = -1, lead = -1, common = 0, core_from = 0, core_to = 0;
    if (G) {
        // bounds of groups in order and within the batch, whatever starts holds
        const int mine = t <= G ? bound(t) : 0, last = G == T && t == 0 ? bound(G) : 0;
        const int lo = scan(mine, s_wave, Largest());
        if (t <= G) s_lo[t] = lo;
        s_from[t] = -1, s_to[t] = 0;   // no member is worked on with others
        __syncthreads();
        if (G == T && t == 0) s_lo[G] = max(last, s_lo[G - 1]);
        __syncthreads();
        if (t < B) {
            int x = 0, y = G;   // the last group that begins at or before t
            while (y - x > 1) {
                const int mid = (x + y) / 2;
                if (s_lo[mid] <= t) x = mid; else y = mid;
            }
            if (t >= s_lo[x] && t < s_lo[x + 1]) {
                group = x, common = max(0, p.shared[x]);
                lead = p.prefix_rows ? p.prefix_rows[x] : row_of(a, s_lo[x]);
                atomicMax(&s_to[x], min(len, common));
            }
        }
        __syncthreads();
        // What is worked on together is what all members attend to, but for those whose tokens end before those that
        // are shared, or whose window begins after them, which go by themselves: so that no token that one
        // attends to, whatever it holds, meets the queries of another that does not.
        const bool together = group >= 0 && begin < s_to[group] && len >= s_to[group];
        if (together) atomicMax(&s_from[group], begin);
        __syncthreads();
        if (together) core_from = s_from[group], core_to = s_to[group];   // begin < s_to of each, so of the largest
    }
    s_own[t].begin = begin, s_own[t].cut = core_to ? core_from - begin : INT32_MAX, s_own[t].skip = core_to - core_from;
    s_own[t].row = row, s_own[t].lead = lead, s_own[t].shared = common, s_own[t].len = len - begin - (core_to - core_from);
    // item t: what group t shares; item G + t: what sequence t has of its own
    struct Item {
        int units, steps, cost;
        int64_t all;
    } item[2];
    int blocks = 0;
    for (int k = 0; k < 2; ++k) {
        Item &i = item[k];
        i.units = i.steps = i.cost = 0;
        if (k == 0 && t < G) {
            const int columns = (s_lo[t + 1] - s_lo[t]) * a.group;
            blocks = (columns + block_columns - 1) / block_columns;
            i.steps = s_from[t] < 0 ? 0 : (s_to[t] - s_from[t] + kStep - 1) / kStep;
            i.units = i.steps ? blocks * a.c.kv_heads : 0;
            if (i.units) i.cost = cost_of(f32, min(columns, block_columns), blocks);
        } else if (k == 1 && t < B) {
            i.steps = (s_own[t].len + kStep - 1) / kStep;
            i.units = i.steps ? a.c.kv_heads * a.head_groups : 0;
            i.cost = cost_of(f32, min(16, a.group), a.head_groups);
        }
        i.all = (int64_t)i.units * i.steps * i.cost;
    }
    auto total_of = [&](int64_t v, int which) {
        v = wave_all(v, Sum());
        if (t % 64 == 0) s_sum[t / 64][which] = v;
    };
    total_of(item[0].all, 0), total_of(item[1].all, 1), total_of((int64_t)item[1].units * item[1].cost, 2);
    __syncthreads();
    int64_t of_groups_all = 0, own_all = 0, own_step = 0;
    for (int w = 0; w < W; ++w) of_groups_all += s_sum[w][0], own_all += s_sum[w][1], own_step += s_sum[w][2];
    // Where what sequences have of their own is much of the work, and short, its tasks are chains of latencies: several units go
    // in one, a part of the waves for each (32 sequences of 256 tokens after 4096 shared ones 44 -> 38 us, 64 of 16 tokens after
    // 3000 64 -> 54; of 2000 tokens after 1 83 -> 90, of 128 tokens after 32768 153 -> 164).
    const int bundle = own_all <= 2 * own_step && 2 * own_all >= of_groups_all ? z.bundle_log2 : 0;
    // The units of a task are worked on side by side: a step of eight takes some 9 us, of 128 columns
    // of a group 5.
    const int64_t per_seq = (int64_t)a.c.kv_heads * a.head_groups, bundles = (per_seq + (1 << bundle) - 1) >> bundle;
    if (bundle) item[1].units = item[1].units ? (int)bundles : 0, item[1].cost *= 2;
    // Of the tasks as they are, since it bounds the number of pieces.
    const int64_t total = of_groups_all + (bundle ? own_all / per_seq * bundles * 2 : own_all);
    // One task for a workgroup, or two of half the cost where these fill the card more evenly: the tasks of groups in all,
    // in rounds of the card, at the cost of the largest.  Two also where what sequences have of their own is a third of
    // the work, whose tasks differ more than the model knows: 60 sequences of up to 4000 own tokens 138 and 117 us, 64 of
    // 1000 after 16000 shared ones 146 and 125, but of 600 after 32768 169 and 190, of 100 in 3 groups of 8000 85 and
    // 98.  Three or four tasks are not better.
    auto pieces_of = [&](const Item &i, int64_t most) {
        // in fp64, which holds these whole numbers, as a division of 64 bits takes a hundred instructions
        return i.units ? max(1, min(i.steps, (int)min(ceil((double)i.steps * i.cost / (double)most), 1e9))) : 0;
    };
    static_assert(kRounds == 2, "");
    int64_t most_of[kRounds], tasks[kRounds], longest[kRounds], few = 0, few_most[2];
    for (int r = 0; r < kRounds; ++r) {
        most_of[r] = max((int64_t)kLeastTask, (int64_t)ceil((double)total / (kGrid * (r + 1))));
        const int n = pieces_of(item[0], most_of[r]);
        tasks[r] = (int64_t)n * item[0].units, longest[r] = n ? (int64_t)((item[0].steps + n - 1) / n) * item[0].cost : 0;
    }
    for (int r = 0; r < kRounds; ++r) tasks[r] = wave_all(tasks[r], Sum()), longest[r] = wave_all(longest[r], Largest());
    // Where even two tasks a workgroup would be small, smaller ones than otherwise, if there is a workgroup for each (32
    // sequences over 4096 shared tokens 36.3 -> 34.4 us, 64 of 8 in 4 groups of 3000 44.4 -> 38.3; with more tasks than
    // workgroups 64 of 64 heads over 3000 53.8 -> 68.5).
    const bool small = total < kGrid * kRounds * kLeastTask;
    if (small) {
        for (int r = 0; r < 2; ++r) {
            few_most[r] = max((int64_t)(kLeastTask * (r + 2) / 4), (int64_t)ceil((double)total / (kGrid * kRounds)));
            for (int k = 0; k < 2; ++k) few += (int64_t)pieces_of(item[k], few_most[r]) * item[k].units << 32 * r;
        }
        few = wave_all(few, Sum());
    }
    __syncthreads();   // the total has been read
    if (t % 64 == 0) {
        int64_t *of = s_sum[t / 64];
        of[0] = tasks[0], of[1] = tasks[1], of[2] = longest[0], of[3] = longest[1], of[4] = few;
    }
    __syncthreads();
    int64_t best = INT64_MAX, most = 1;
    for (int r = 0; r < kRounds; ++r) {
        int64_t n = 0, l = 0;
        for (int w = 0; w < W; ++w) n += s_sum[w][r], l = max(l, s_sum[w][2 + r]);
        const int64_t time = max((n + kGrid - 1) / kGrid * (l + kTaskCost), total / kGrid + kTaskCost * (r + 1));
        if (time < best || 2 * own_all >= of_groups_all) best = time, most = most_of[r];
    }
    if (small) {
        int64_t n = 0;
        for (int w = 0; w < W; ++w) n += s_sum[w][4];
        if (n >> 32 <= kGrid) most = few_most[1];
        if ((uint32_t)n <= kGrid) most = few_most[0];
    }
    // numbers of tasks: those of groups, then those of sequences, both in one scan
    const int n0 = pieces_of(item[0], most), n1 = pieces_of(item[1], most);
    const int64_t count = (int64_t)(n0 * item[0].units) << 32 | (uint32_t)(n1 * item[1].units);
    const int64_t upto = scan(count, &s_sum[0][0], Sum());
    if (t == T - 1) s_all = upto;
    __syncthreads();
    const int of_groups = (int)(s_all >> 32), before = of_groups + (int)(uint32_t)s_all;
    const int first_task[2] = {(int)((upto - count) >> 32), of_groups + (int)(uint32_t)(upto - count)};
    if (t < G) s_task[t] = first_task[0], s_pieces[t] = n0, s_steps[t] = item[0].steps;
    if (t < B) s_task[G + t] = first_task[1], s_pieces[G + t] = n1, s_steps[G + t] = item[1].steps;
    if (t == 0) {
        s_task[G + B] = before;
        space.head->shared = of_groups, space.head->tasks = before, space.head->next = min(before, kGrid), space.head->bundle = bundle;
        for (int i = 0; i < 4; ++i) space.head->zero[i] = 0;
    }
    __syncthreads();
    if (t < B) {
        Member m = {0, 0, 0, 0, first_task[1] - of_groups, n1, {0, 0}};
        if (core_to) {
            m.task = s_task[group], m.pieces = s_pieces[group], m.place = t - s_lo[group];
            m.blocks = ((s_lo[group + 1] - s_lo[group]) * a.group + block_columns - 1) / block_columns;
        }
        space.member[t] = m;
    }
    for (int task = t; task < before; task += T) {
        int x = 0, y = G + B;   // the last item that begins at or before the task, which has tasks
        while (y - x > 1) {
            const int mid = (x + y) / 2;
            if (s_task[mid] <= task) x = mid; else y = mid;
        }
        const int n = s_pieces[x], steps = s_steps[x], in = task - s_task[x];
        Task k;
        int piece, end;
        if (x < G) {   // by head, piece, block of columns: what is read together is worked on together
            const int all = (s_lo[x + 1] - s_lo[x]) * a.group, nb = (all + block_columns - 1) / block_columns;
            piece = in / nb % n, k.j = in / nb / n, k.first = s_lo[x], k.c0 = in % nb * block_columns;
            k.columns = min(block_columns, all - k.c0), k.units = 0;
            k.row = k.lead = p.prefix_rows ? p.prefix_rows[x] : row_of(a, k.first);
            k.shared = 0, k.begin = s_from[x], k.cut = INT32_MAX, k.skip = 0, end = s_to[x] - s_from[x];
        } else {
            const int b = x - G;
            piece = in % n, k.j = in / n << bundle, k.first = b, k.c0 = k.columns = 0;
            k.units = min(1 << bundle, a.c.kv_heads * a.head_groups - k.j);
            k.row = s_own[b].row, k.lead = s_own[b].lead, k.shared = s_own[b].shared;
            k.begin = s_own[b].begin, k.cut = s_own[b].cut, k.skip = s_own[b].skip, end = s_own[b].len;
        }
        const int each_steps = steps / n, more = steps - each_steps * n;   // the first `more` pieces have one step more
        k.from = (each_steps * piece + min(piece, more)) * kStep;
        k.to = min(end, (each_steps * (piece + 1) + min(piece + 1, more)) * kStep);
        k.number = task;
        // The first tasks go by workgroup: those that read the same to the same XCD, whose L2 then holds it.
        const int each = (min(before, kGrid) + 7) / 8;
        space.task[task < kGrid ? task % each * 8 + task / each : task] = k;
    }
    // workgroups for which there is none
    const int each = (min(before, kGrid) + 7) / 8;
    for (int i = t; i < kGrid; i += T)
        if (i / 8 >= each || i % 8 * each + i / 8 >= before) space.task[i].number = -1;
}

// ---- up to 32 columns --------------------------------------------------------------------------------

template <typename E, int DP, int N, int WAVES> struct Narrow {
    static constexpr int ROW = DP + 4;
    int64_t place[kTile];
    float m[WAVES][16 * N], l[WAVES][16 * N];
    union {
        __attribute__((aligned(16))) E q[16 * N][DP + 16 / sizeof(E)];
        __attribute__((aligned(16))) float o[WAVES][16 * N][ROW];
    };
};

// Largest score and sum of a softmax, of a lane's column.  The reference is not the maximum but within 2^6 of it, or
// above: it moves only where some score passes it by so much, which costs a vote a step instead of two
// exchanges and a product for every output.
constexpr float kPast = 6.f;

// Element offset of token number i of a task in a plane, or -1 where there is none.
__device__ __forceinline__ int64_t place_in(const AttnArgs &a, const Task &k, int i) {
    if (i >= k.to) return -1;
    const int t = k.begin + i + (i >= k.cut ? k.skip : 0);
    return place_of(a.c, a.table, t < k.shared ? k.lead : k.row, a.seqs, a.width, t);
}

// Queries of a task's columns to LDS, put(column, dimension, value), 0 past the columns and head_dim: every thread
// has a column, so that what divides is done once.
template <typename E, int COLUMNS, int DP, int THREADS, typename P>
__device__ __forceinline__ void stage_queries(const AttnArgs &a, const Task &k, P put) {
    const Scale scale(a.scale);
    constexpr int EACH = THREADS / COLUMNS, AHEAD = DP / EACH < 16 ? DP / EACH : 16;   // dimensions at a time; loads under way
    const int c = threadIdx.x % COLUMNS, at = k.c0 + min(c, k.columns - 1), s = at / a.group, D = a.c.head_dim;
    const E *q = (const E *)a.q + (k.first + s) * a.qs.seq + (k.j * a.group + at - s * a.group) * a.qs.head;
    for (int d0 = threadIdx.x / COLUMNS; d0 < DP; d0 += EACH * AHEAD) {
        E v[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) v[i] = q[min(d0 + i * EACH, D - 1) * a.qs.dim];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) put(c, d0 + i * EACH, c < k.columns && d0 + i * EACH < D ? scale.of(v[i]) : (E)0);
    }
}

// Columns c0 .. of key head j, from sequence `first` on.
struct Columns {
    int j, first, c0, columns;
};
__device__ __forceinline__ Columns unit_of(const AttnArgs &a, const Task &k, int unit) {
    if (!k.units) return {k.j, k.first, k.c0, k.columns};
    const int u = k.j + min(unit, k.units - 1), j = u / a.head_groups, c0 = (u - j * a.head_groups) * 16;
    return {j, k.first, c0, min(16, a.group - c0)};
}
// A column's query as it was laid out; past the columns that of the last.
template <int DP, typename E> __device__ __forceinline__ const E *query_of(const AttnArgs &a, const Columns &k, const E *laid, int c) {
    const int at = k.c0 + min(c, k.columns - 1), s = at / a.group;
    return laid + ((int64_t)(k.first + s) * a.heads + k.j * a.group + at - s * a.group) * DP;
}

// N sixteens of columns over a task's tokens, or 1 << bundle units of 16, each by a part of the waves.
// finish(unit, column, d, output, reference, sum) takes what comes of them, joined over the waves.
// `laid`: queries as lay_queries leaves them, or none.
template <typename E, int DP, bool FULL, int N, int WAVES, typename F>
__device__ __forceinline__ void columns_narrow(const AttnArgs &a, Narrow<E, DP, N, WAVES> &sh, const Task &k, int bundle, const E *laid, F finish) {
    typedef Step<E, DP> St;
    constexpr int TOK = St::TOK, TT = TOK / 4, NT = TOK / 16, VW = St::VW, NV = St::NV, THREADS = 64 * WAVES;
    const int D = a.c.head_dim, wave = uni(threadIdx.x / 64);
    int lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));   // what goes by the lane is worked out again for each task, not held in registers
    const int r = lane % 16, quad = lane / 16;
    const int each = WAVES >> bundle, unit = wave / each, first = wave - unit * each;   // waves of a unit
    const Columns mine = unit_of(a, k, unit);
    const int j = uni(mine.j);
    const E *keys = (const E *)a.keys + j * a.c.head_stride, *values = (const E *)a.values + j * a.c.head_stride;
    const Scale scale(a.scale);

    St st;
    typename St::Quad q[N][St::NK];
    f32x4 acc[N][NV][VW];
    float m[N], ref[N], l[N];   // ref: m, or 0 before any
#pragma unroll
    for (int n = 0; n < N; ++n) {
        m[n] = -INFINITY, ref[n] = l[n] = 0.f;
#pragma unroll
        for (int h = 0; h < NV; ++h)
#pragma unroll
            for (int i = 0; i < VW; ++i) acc[n][h][i] = (f32x4){0, 0, 0, 0};
    }

    for (int base = k.from; base < k.to; base += kTile) {
        const int n = min(kTile, k.to - base), padded = (n + TOK - 1) / TOK * TOK;
        if (base > k.from) __syncthreads();   // places of the tile before are no longer read
        for (int t = threadIdx.x; t < padded; t += THREADS)
            sh.place[t] = place_in(a, k, base + t);
        if (base == k.from && laid) {   // queries come while the places do
#pragma unroll
            for (int c = 0; c < N; ++c) St::load_q(q[c], query_of<DP>(a, mine, laid, c * 16 + r), quad);
        } else if (base == k.from)
            stage_queries<E, 16 * N, DP, THREADS>(a, k, [&](int c, int d, E v) { sh.q[c][d] = v; });
        __syncthreads();
        if (base == k.from && !laid)
#pragma unroll
            for (int c = 0; c < N; ++c) St::load_q(q[c], sh.q[c * 16 + r], quad);
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
        auto softmax = [&]() __attribute__((always_inline)) {
            const bool whole = !__any(dead != 0);
            if (!whole) {
#pragma unroll
                for (int c = 0; c < N; ++c)
#pragma unroll
                    for (int i = 0; i < TT; ++i)
                        if (dead >> i & 1) s[c][i] = -INFINITY;
                st.clear_v(dead);
            }
            float top[N];
            bool past = false;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                top[c] = s[c][0];
#pragma unroll
                for (int i = 1; i < TT; ++i) top[c] = fmaxf(top[c], s[c][i]);
                top[c] *= scale.by;
                past |= top[c] > m[c] + kPast;
            }
            if (__any(past))
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    float to = fmaxf(top[c], __shfl_xor(top[c], 16));
                    to = fmaxf(m[c], fmaxf(to, __shfl_xor(to, 32)));
                    const float keep = m[c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[c] - to);
                    m[c] = to, ref[c] = to == -INFINITY ? 0.f : to, l[c] *= keep;
#pragma unroll
                    for (int h = 0; h < NV; ++h)
#pragma unroll
                        for (int i = 0; i < VW; ++i) acc[c][h][i] *= keep;
                }
#pragma unroll
            for (int c = 0; c < N; ++c) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < TT; ++i) {
                    s[c][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][i], scale.by, -ref[c]));
                    sum += s[c][i];
                }
                l[c] += sum;
            }
            st.template outputs<N>(s, acc);
        };
        int s0 = first * TOK;
        if (s0 < padded && (unit == 0 || unit < k.units)) {
            load_k(s0);
            load_v(s0);
            for (;;) {
#pragma unroll
                for (int c = 0; c < N; ++c) st.template scores<FULL>(q[c], s[c], D);
                const int next = s0 + each * TOK;
                if (next >= padded) break;
                load_k(next);
                softmax();
                load_v(next);
                s0 = next;
            }
            softmax();
        }
    }

    __syncthreads();   // queries are no longer read: their place is taken
#pragma unroll
    for (int c = 0; c < N; ++c) {
        l[c] += __shfl_xor(l[c], 16);
        l[c] += __shfl_xor(l[c], 32);
        if (quad == 0) sh.m[wave][c * 16 + r] = m[c], sh.l[wave][c * 16 + r] = l[c];
        if (c * 16 + r < mine.columns)
#pragma unroll
            for (int h = 0; h < NV; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < VW; v += 4)
                        *(f32x4 *)&sh.o[wave][c * 16 + r][h * 16 * VW + (quad * 4 + i) * VW + v] =
                            (f32x4){acc[c][h][v][i], acc[c][h][v + 1][i], acc[c][h][v + 2][i], acc[c][h][v + 3][i]};
    }
    __syncthreads();
    const int columns = k.units ? k.units * 16 : k.columns;
    for (int i = threadIdx.x; i < columns * DP; i += THREADS) {
        const int of = k.units ? i / (16 * DP) : 0, c = i / DP - of * 16, d = i % DP;
        if (d >= D || c >= unit_of(a, k, of).columns) continue;
        float top = -INFINITY, sum = 0.f, o = 0.f;
        for (int w = of * each; w < (of + 1) * each; ++w) top = fmaxf(top, sh.m[w][c]);
        const float ref = top == -INFINITY ? 0.f : top;
        for (int w = of * each; w < (of + 1) * each; ++w) {
            const float f = __builtin_amdgcn_exp2f(sh.m[w][c] - ref);
            sum += sh.l[w][c] * f, o += sh.o[w][c][d] * f;
        }
        finish(of, c, d, o, top, sum);
    }
    __syncthreads();   // the next task writes these arrays
}

// ---- more columns ------------------------------------------------------------------------------------

// Keys and values of 128 tokens, twice: one is worked on while the other comes.  Rows of DP dimensions, in which 16
// bytes lie at the place that the row turns them to: sixteen lanes that read a piece of sixteen rows, or 32 bytes of
// four, then meet all banks.
template <int DP> struct Wide {
    static constexpr int ROW = DP + 4;
    uint16_t stage[2][2][kStep * DP];   // [which][keys, values]
    int64_t place[2][kTile];
    int holes[2];                       // whether a tile has a token that holds nothing
    float m[8][32], l[8][32];
    __device__ __forceinline__ float *joined(int wave) { return (float *)stage + wave * 32 * ROW; }
};
template <int DP> __device__ __forceinline__ int turn_of(int row) { return DP == 128 ? row & 15 : row >> 1 & 7; }

// N times 16 bytes from each lane's sources to LDS, byte address base + 1024 i + 16 lane; counted as N loads of the
// wave.  The offset moves source and destination alike.
template <int N> __device__ __forceinline__ void copy16(const char *const *src, uint32_t base) {
    uint32_t saved;
    static_assert(N == 2 || N == 4, "");
    if constexpr (N == 2)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %1, off\n\tglobal_load_lds_dwordx4 %2, off offset:1024\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved) : "v"(src[0]), "v"(src[1] - 1024), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %1, off\n\tglobal_load_lds_dwordx4 %2, off offset:1024\n\t"
                     "global_load_lds_dwordx4 %3, off offset:2048\n\tglobal_load_lds_dwordx4 %4, off offset:%6\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved) : "v"(src[0]), "v"(src[1] - 1024), "v"(src[2] - 2048), "v"(src[3] - 3 * 1024), "s"(base), "n"(3 * 1024)
                     : "memory");
}

// CW: waves that share the columns, 32 each; the 8 / CW sets of these share the tokens of a stage.  Of 256 columns over 32
// tokens the two waves of a SIMD take 2129 cycles (48 MFMA by themselves 1500, 160 VALU instructions 1227), 153 thousand
// for the 18 stages of a task of 64 sequences over 32768 tokens, which takes some 220 thousand: the others, in which
// stages begin and end and wait for each other, have not been accounted for one by one.  One bf16 for a probability
// would save an eighth of the time, and half of its bits.  A priority for either wave or keys of the next step read ahead
// save nothing.
template <int DP, bool FULL, int CW>
__device__ __forceinline__ void columns_wide(const AttnArgs &a, Wide<DP> &sh, const Task &k, const uint16_t *laid, const void *zero,
                                             const Parts &parts, int64_t task) {
    typedef uint16_t E;
    constexpr int NC = DP / 32, ND = DP / 16, GR = DP / 8, SETS = 8 / CW, TOKENS = kStep / SETS;
    const int D = a.c.head_dim, wave = uni(threadIdx.x / 64), set = wave / CW, c_wave = wave % CW * 32;
    int lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));
    const int r = lane % 16, quad = lane / 16;
    const E *keys = (const E *)a.keys + k.j * a.c.head_stride, *values = (const E *)a.values + k.j * a.c.head_stride;
    const Scale scale(a.scale);
    const uint32_t stage0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)sh.stage;

    auto fill_places = [&](int tile, const int64_t (&at)[kTile / 512]) {
        bool hole = false;
#pragma unroll
        for (int i = 0; i < kTile / 512; ++i) {
            const int t = threadIdx.x + 512 * i;
            sh.place[tile % 2][t] = at[i], hole |= at[i] < 0 && k.from + tile * kTile + t < k.to;
        }
        if (hole) sh.holes[tile % 2] = 1;
    };
    // A wave copies 1 KB at a time of a stage's keys and values, each lane 16 bytes of the row that they belong to.
    constexpr int ROWS = 64 / GR, N = kStep / ROWS / 8;   // rows of a copy, copies of a wave
    auto copy = [&](int s) {
        const uint32_t to = (uint32_t)uni((int)(stage0 + (uint32_t)(s % 2 * 2 * kStep * DP * 2) + wave * N * 1024));
        const int64_t *place = &sh.place[s * kStep / kTile % 2][s * kStep % kTile + wave * N * ROWS + lane / GR];
        int64_t at[N];
        bool all = true;
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = place[i * ROWS], all &= at[i] >= 0;
        const char *ks[N], *vs[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int g = lane % GR ^ turn_of<DP>(i * ROWS + lane / GR);   // of the wave's rows, which begin at a multiple of 16
            ks[i] = (const char *)(keys + g * 8) + 2 * at[i], vs[i] = (const char *)(values + g * 8) + 2 * at[i];
            if (!FULL && g * 8 >= D) ks[i] = vs[i] = (const char *)zero;
        }
        if (__any(!all))
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (at[i] < 0) ks[i] = vs[i] = (const char *)zero;
        copy16<N>(ks, to);
        copy16<N>(vs, to + kStep * DP * 2);
    };

    const int stages = (k.to - k.from + kStep - 1) / kStep;
    if (threadIdx.x < 2) sh.holes[threadIdx.x] = 0;
    __syncthreads();
    int64_t ahead[kTile / 512];
#pragma unroll
    for (int i = 0; i < kTile / 512; ++i) ahead[i] = place_in(a, k, k.from + threadIdx.x + 512 * i);
    fill_places(0, ahead);
    __syncthreads();
    copy(0);
    u32x4 q[2][NC];
    f32x4 acc[2][ND];
    float m[2], ref[2], l[2];   // ref: m, or 0 before any
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int c = c_wave + n * 16 + r;
#pragma unroll
        for (int i = 0; i < NC; ++i) q[n][i] = *(const u32x4 *)(query_of<DP>(a, {k.j, k.first, k.c0, k.columns}, laid, c) + i * 32 + quad * 8);
        m[n] = -INFINITY, ref[n] = l[n] = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[n][d] = (f32x4){0, 0, 0, 0};
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    // where a lane reads in a stage: its part of a key, and its four tokens' values
    uint32_t k_at[NC], v_at[ND];
#pragma unroll
    for (int i = 0; i < NC; ++i) k_at[i] = stage0 + (r * DP + ((i * 4 + quad) ^ turn_of<DP>(r)) * 8) * 2;
#pragma unroll
    for (int d = 0; d < ND; ++d) {   // of sixteen lanes, lane i names token i / 4 and four dimensions, and gets one dimension of four tokens
        const int row = 4 * quad + r / 4;
        v_at[d] = stage0 + (kStep * DP + row * DP + ((2 * d + r % 4 / 2) ^ turn_of<DP>(row)) * 8 + r % 2 * 4) * 2;
    }
    for (int s = 0; s < stages; ++s) {
        // the next stage comes, and with a tile's first stage the places of the next tile
        const bool more_places = s * kStep % kTile == 0 && (s * kStep / kTile + 1) * kTile < k.to - k.from;
        if (s + 1 < stages) copy(s + 1);
        if (more_places)
#pragma unroll
            for (int i = 0; i < kTile / 512; ++i) ahead[i] = place_in(a, k, k.from + (s * kStep / kTile + 1) * kTile + threadIdx.x + 512 * i);
        uint32_t ka[NC], va[ND];
#pragma unroll
        for (int i = 0; i < NC; ++i) ka[i] = k_at[i] + (uint32_t)((s % 2 * 2 * kStep + set * TOKENS) * DP * 2);
#pragma unroll
        for (int d = 0; d < ND; ++d) va[d] = v_at[d] + (uint32_t)((s % 2 * 2 * kStep + set * TOKENS) * DP * 2);
        const bool holes = sh.holes[s * kStep / kTile % 2];
#pragma unroll 1
        for (int t0 = set * TOKENS; t0 < (set + 1) * TOKENS; t0 += 32) {
            const int token = k.from + s * kStep + t0;
            if (token >= k.to) break;
            float p[2][8];
            // Scores of 32 tokens: rows are tokens, columns queries.  All reads of a step go out before what waits for them.
            u32x4 kv[2][NC];
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) kv[t][i] = *(lds_u32x4 *)(uintptr_t)(ka[i] + 16 * t * DP * 2);
            __builtin_amdgcn_sched_barrier(0);
            f32x4 c4[2][2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n) c4[n][t] = (f32x4){0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int n = 0; n < 2; ++n)
                        c4[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kv[t][i]), as_bf16x8(q[n][i]), c4[n][t], 0, 0, 0);
            u32x2 w[ND][2];
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    w[d][t] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(va[d] + 16 * t * DP * 2)));
#pragma unroll
            for (int i = 0; i < NC; ++i) ka[i] += 32 * DP * 2;
#pragma unroll
            for (int d = 0; d < ND; ++d) va[d] += 32 * DP * 2;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[n][4 * t + i] = c4[n][t][i];
            // tokens that hold nothing, whose keys and values came as 0: their scores are -Inf, and so what they weigh 0
            if (holes || token + 32 > k.to)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (sh.place[s * kStep / kTile % 2][(s * kStep + t0 + 16 * (i / 4) + 4 * quad + i % 4) % kTile] < 0)
                        p[0][i] = p[1][i] = -INFINITY;
            float top[2];
            bool past = false;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                top[n] = p[n][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top[n] = fmaxf(top[n], p[n][i]);
                top[n] *= scale.by;
                past |= top[n] > m[n] + kPast;
            }
            if (__any(past))
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    float to = fmaxf(top[n], __shfl_xor(top[n], 16));
                    to = fmaxf(m[n], fmaxf(to, __shfl_xor(to, 32)));
                    const float keep = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - to);
                    m[n] = to, ref[n] = to == -INFINITY ? 0.f : to, l[n] *= keep;
#pragma unroll
                    for (int d = 0; d < ND; ++d) acc[n][d] *= keep;
                }
            u32x4 b[2][2];   // a probability is the sum of two bf16, as in k_attn
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[n][i], scale.by, -ref[n]));
                    sum += p[n][i];
                }
                l[n] += sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    b[n][0][i] = pack_bf16(p[n][2 * i], p[n][2 * i + 1]);
                    b[n][1][i] = pack_bf16(p[n][2 * i] - bf16_to_f32(b[n][0][i]), p[n][2 * i + 1] - __uint_as_float(b[n][0][i] & 0xffff0000u));
                }
            }
            // outputs: rows are dimensions
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const bf16x8 v = as_bf16x8((u32x4){w[d][0].x, w[d][0].y, w[d][1].x, w[d][1].y});
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int n = 0; n < 2; ++n) acc[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, as_bf16x8(b[n][i]), acc[n][d], 0, 0, 0);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the copies have landed
        if (more_places) {
            const int tile = s * kStep / kTile + 1;
            if (threadIdx.x == 0) sh.holes[tile % 2] = 0;
            __syncthreads();
            fill_places(tile, ahead);
        }
        __syncthreads();
    }

    // join the sets, then to the parts: a lane has four dimensions of a column
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (SETS > 1 && quad == 0) sh.m[wave][n * 16 + r] = m[n], sh.l[wave][n * 16 + r] = l[n];
        if (SETS > 1 && set > 0)
#pragma unroll
            for (int d = 0; d < ND; ++d) *(f32x4 *)&sh.joined(wave - CW)[(n * 16 + r) * Wide<DP>::ROW + d * 16 + quad * 4] = acc[n][d];
    }
    if (SETS > 1) __syncthreads();
    if (set == 0)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int c = c_wave + n * 16 + r;
            if (SETS > 1) {
                float to = m[n];
                for (int w = wave + CW; w < 8; w += CW) to = fmaxf(to, sh.m[w][n * 16 + r]);
                const float ref = to == -INFINITY ? 0.f : to, keep = __builtin_amdgcn_exp2f(m[n] - ref);
                l[n] *= keep;
#pragma unroll
                for (int d = 0; d < ND; ++d) acc[n][d] *= keep;
                for (int w = wave + CW; w < 8; w += CW) {
                    const float f = __builtin_amdgcn_exp2f(sh.m[w][n * 16 + r] - ref);
                    l[n] += sh.l[w][n * 16 + r] * f;
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        acc[n][d] += *(const f32x4 *)&sh.joined(w - CW)[(n * 16 + r) * Wide<DP>::ROW + d * 16 + quad * 4] * f;
                }
                m[n] = to;
            }
            if (c >= k.columns) continue;
            const int64_t at = parts.at(task, c);
#pragma unroll
            for (int d = 0; d < ND; ++d)
                if (FULL || d * 16 + quad * 4 < D) *(f32x4 *)&parts.o[at * D + d * 16 + quad * 4] = acc[n][d];
            if (quad == 0) parts.m[at] = m[n], parts.l[at] = l[n];
        }
    __syncthreads();   // the next task writes these arrays
}

// ---- the kernels -------------------------------------------------------------------------------------

template <typename E, int DP> struct Shared {
    static constexpr int WAVES = kTaskWaves<DP>;
    static constexpr bool WIDE = kColumns<E, DP> > 32;
    struct Nothing {};
    union {
        Narrow<E, DP, 1, WAVES> one;
        Narrow<E, DP, 2, WAVES> two;
        std::conditional_t<WIDE, Wide<DP == 256 ? 128 : DP>, Nothing> wide;
    };
    int next;
    __device__ Shared() {}
};

template <typename E, int DP, bool FULL>
__global__ __launch_bounds__(64 * kTaskWaves<DP>, kTaskWaves<DP> / 4) void k_prefix(PrefixArgs p, Sizes z) {
    __shared__ Shared<E, DP> sh;
    const AttnArgs &a = p.a;
    const Space space = space_of(a.workspace, z, a.batch, a.c.head_dim);
    const int tasks = uni(space.head->tasks), shared = uni(space.head->shared), bundle = uni(space.head->bundle);
    const E *laid = (const E *)space.q;
    int slot = blockIdx.x;   // of the task; later ones have their own number's
    for (;;) {
        const Task *at = space.task + slot;
        Task k;
        k.j = uni(at->j), k.first = uni(at->first), k.c0 = uni(at->c0), k.columns = uni(at->columns), k.from = uni(at->from);
        k.to = uni(at->to), k.row = uni(at->row), k.lead = uni(at->lead), k.shared = uni(at->shared), k.begin = uni(at->begin);
        k.cut = uni(at->cut), k.skip = uni(at->skip), k.number = uni(at->number), k.units = uni(at->units);
        if (k.number < 0) return;
        if (tasks > kGrid && threadIdx.x == 0) sh.next = atomicAdd(&space.head->next, 1);
        const bool common = k.number < shared;
        const Parts parts = common ? space.shared : space.own;
        const int64_t number = common ? k.number : k.number - shared;
        auto finish = [&](int unit, int c, int d, float o, float m, float l) {
            const int64_t i = parts.at(common ? number : (number << bundle) + unit, c);
            parts.o[i * a.c.head_dim + d] = o;
            if (d == 0) parts.m[i] = m, parts.l[i] = l;
        };
        if (k.columns <= 16) {   // or units
            columns_narrow<E, DP, FULL, 1, kTaskWaves<DP>>(a, sh.one, k, k.units ? bundle : 0, laid, finish);
        } else if (k.columns <= 32 || !Shared<E, DP>::WIDE) {
            columns_narrow<E, DP, FULL, 2, kTaskWaves<DP>>(a, sh.two, k, 0, laid, finish);
        } else if constexpr (Shared<E, DP>::WIDE) {
            const void *zero = space.head->zero;
            if (k.columns <= 64)
                columns_wide<DP, FULL, 2>(a, sh.wide, k, laid, zero, parts, number);
            else if (k.columns <= 128)
                columns_wide<DP, FULL, 4>(a, sh.wide, k, laid, zero, parts, number);
            else
                columns_wide<DP, FULL, 8>(a, sh.wide, k, laid, zero, parts, number);
        }
        if (tasks <= kGrid) return;
        slot = uni(sh.next);
        if (slot >= tasks) return;
        __syncthreads();   // read before the next one is written
    }
}

// Joins the tasks of a query head, those of its group and its own: 4 dimensions a thread, eight tasks at a time.
constexpr int kMostJoined = 512;   // whose factors are held at a time
template <typename E>
__global__ __launch_bounds__(256) void k_prefix_join(PrefixArgs p, Sizes z, int block_columns) {
    constexpr int LANES = 32, GROUPS = 256 / LANES;
    __shared__ float s_f[kMostJoined], s_top[4], s_sum[4];
    __shared__ f32x4 s_o[GROUPS][LANES];
    __shared__ int s_nan, s_kinds[4 * LANES];
    const AttnArgs &a = p.a;
    const int h = blockIdx.x % a.heads, b = blockIdx.x / a.heads, t = threadIdx.x, D = a.c.head_dim;
    const int j = h / a.group, hh = h - j * a.group;
    const Space space = space_of(a.workspace, z, a.batch, D);
    const Member me = space.member[b];
    const int column = me.place * a.group + hh, block = column / block_columns;
    const int n = me.pieces + me.own_pieces, unit = j * a.head_groups + hh / 16, bundle = space.head->bundle;
    auto at = [&](int k, Parts *parts) {
        const bool common = k < me.pieces;
        *parts = common ? space.shared : space.own;
        return common ? space.shared.at(me.task + (int64_t)(j * me.pieces + k) * me.blocks + block, column - block * block_columns)
                      : space.own.at(((me.own_task + (int64_t)(unit >> bundle) * me.own_pieces + k - me.pieces) << bundle)
                                         + (unit & ((1 << bundle) - 1)), hh % 16);
    };
    auto finite = [](float top) { return top == -INFINITY ? 0.f : top; };   // what is taken off: -Inf - -Inf is none
    float top = -INFINITY, sum = 0.f;
    for (int k = t; k < n; k += 256) {
        Parts parts;
        const int64_t i = at(k, &parts);
        const float m = parts.m[i], l = parts.l[i], to = fmaxf(top, m), ref = finite(to);
        if (k < kMostJoined) s_f[k] = m;
        sum = sum * __builtin_amdgcn_exp2f(top - ref) + l * __builtin_amdgcn_exp2f(m - ref);
        top = to;
    }
    float all = top;
    for (int i = 1; i < 64; i *= 2) all = fmaxf(all, __shfl_xor(all, i));
    sum *= __builtin_amdgcn_exp2f(top - finite(all));
    for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
    if (t % 64 == 0) s_top[t / 64] = all, s_sum[t / 64] = sum;
    if (t < 4 * LANES) s_kinds[t] = 0;
    if (t == 0) s_nan = 0;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    const float ref = finite(top);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += s_sum[w] * __builtin_amdgcn_exp2f(s_top[w] - ref);
    const int from = blockIdx.y * (4 * LANES), d = from + t % LANES * 4;
    f32x4 v = {0, 0, 0, 0};
    for (int k = t / LANES; k < n; k += GROUPS) {
        Parts parts;
        const int64_t i = at(k, &parts);
        const float m = k < kMostJoined ? s_f[k] : parts.m[i];
        v += *(const f32x4 *)(parts.o + i * D + min(d, D - 4)) * __builtin_amdgcn_exp2f(m - ref);
    }
    s_o[t / LANES][t % LANES] = v;
    if (any_nan(v)) s_nan = 1;
    __syncthreads();
    if (__builtin_expect(s_nan && sum == sum, 0)) {   // over what the sequence attends to, in a row
        const PrefixArgs &again = argument_again<PrefixArgs>();
        const AttnArgs &args = again.a;
        const int lane = t % LANES;
        Task k;
        k.row = row_of(args, b), k.to = len_of(args, k.row), k.begin = args.window && k.to > args.window ? k.to - args.window : 0;
        k.to -= k.begin, k.cut = INT32_MAX, k.skip = k.shared = 0, k.lead = -1;
        for (int g = 0; g < again.groups; ++g)
            if (const int lo = again.starts[g]; lo >= 0 && lo <= b && b < again.starts[g + 1])
                k.shared = again.shared[g], k.lead = again.prefix_rows ? again.prefix_rows[g] : row_of(args, lo);
        kinds_of<4, 4>((const E *)args.values + j * args.c.head_stride + min(d, D - 4), k.to, t / LANES, GROUPS,
                       [&](int i) { return place_in(args, k, i); },
                       [&](int e, int found) {
                           if (found) atomicOr(&s_kinds[4 * lane + e], found);
                           return *(volatile int *)&s_kinds[4 * lane + e];
                       });
        __syncthreads();
    }
    const int dim = from + t;
    if (t >= 4 * LANES || dim >= D) return;
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) o += ((const float *)s_o[i])[t];
    if (o != o && sum == sum) o = told_by(s_kinds[t]);
    ((E *)a.y)[b * a.ys.seq + h * a.ys.head + dim * a.ys.dim] = from_f32<E>(sum == 0.f ? 0.f : o / sum);
    if (dim == 0 && a.lse) a.lse[(int64_t)b * a.heads + h] = (ref + log2f(sum)) * kLn2;
}

// A workgroup for up to 16 query heads of a key head of a sequence.
template <typename E, int DP, bool FULL, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP == 256 ? 1 : 2) void k_prefix_short(PrefixArgs p) {
    __shared__ Narrow<E, DP, 1, WAVES> sh;
    const AttnArgs &a = p.a;
    const int per_seq = a.c.kv_heads * a.head_groups, b = blockIdx.x / per_seq, u = blockIdx.x - b * per_seq, lane = threadIdx.x % 64;
    Task k;
    k.row = uni(row_of(a, b)), k.j = u / a.head_groups, k.first = b, k.c0 = (u - k.j * a.head_groups) * 16;
    k.columns = min(16, a.group - k.c0);
    k.units = 0, k.begin = k.from = 0, k.to = uni(len_of(a, k.row)), k.cut = INT32_MAX, k.skip = 0, k.shared = 0, k.lead = -1;
    if (a.window && k.to > a.window) k.begin = k.to - a.window, k.to = a.window;
    for (int g0 = 0; g0 < p.groups; g0 += 64) {
        const int g = g0 + lane;
        const int lo = g < p.groups ? p.starts[g] : 0, hi = g < p.groups ? p.starts[g + 1] : 0;
        const uint64_t hit = __ballot(lo >= 0 && b >= lo && b < hi);
        if (!hit) continue;
        const int at = __ffsll((unsigned long long)hit) - 1;
        k.shared = uni(p.shared[g0 + at]);
        k.lead = uni(p.prefix_rows ? p.prefix_rows[g0 + at] : row_of(a, __shfl(lo, at)));
        break;
    }
    if (k.from >= k.to) {   // no tokens
        for (int i = threadIdx.x; i < k.columns * a.c.head_dim; i += 64 * WAVES) {
            const int c = i / a.c.head_dim, h = k.j * a.group + k.c0 + c, d = i - c * a.c.head_dim;
            ((E *)a.y)[b * a.ys.seq + h * a.ys.head + d * a.ys.dim] = (E)0;
            if (d == 0 && a.lse) a.lse[(int64_t)b * a.heads + h] = -INFINITY;
        }
        return;
    }
    int kinds = 0;
    static_assert(64 * WAVES % DP == 0, "");
    columns_narrow<E, DP, FULL, 1, WAVES>(a, sh, k, 0, (const E *)nullptr, [&](int, int c, int d, float o, float m, float l) {
        if (__builtin_expect(o != o && l == l, 0)) {   // d is the same for all of a thread's outputs
            if (!kinds)
                kinds_of<1, 8>((const E *)a.values + k.j * a.c.head_stride + d, k.to, 0, 1, [&](int i) { return place_in(a, k, i); },
                               [&](int, int found) { return kinds |= found; });
            o = told_by(kinds);
        }
        const int h = k.j * a.group + k.c0 + c;
        ((E *)a.y)[b * a.ys.seq + h * a.ys.head + d * a.ys.dim] = from_f32<E>(l == 0.f ? 0.f : o / l);
        if (d == 0 && a.lse) a.lse[(int64_t)b * a.heads + h] = ((m == -INFINITY ? 0.f : m) + log2f(l)) * kLn2;
    });
}

// Sequences of few tokens take one kernel, in which each reads what it shares by itself: in tables of 1000 tokens 8
// sequences of 8 key heads 14.7 us and by a plan 25.4, 32 sequences 16.4 and 30, 64 of 64 query heads 28 and 43.  Of 2100
// tokens 4 sequences 27 and 25, but 32 sequences, which fill the card, 29 and 32, 64 with nothing shared 61 and 73; of
// 3256 tokens 32 sequences 41 and 33.
constexpr int64_t kShort = 1024;
bool is_short(const CacheArgs &c, int batch, int heads, int64_t tokens) {
    const int64_t units = (int64_t)batch * c.kv_heads * ((heads / c.kv_heads + 15) / 16);
    return tokens <= (units >= 128 ? 2 : 1) * kShort;
}

template <typename E, int DP, bool FULL> hipError_t run(const PrefixArgs &p, bool few, hipStream_t st) {
    const AttnArgs &a = p.a;
    if (few) {
        // Eight waves where each has a CU for itself, unless a wave's registers ask for a SIMD: 132 workgroups of fp32 30.9 ->
        // 26.5 us, 128 and 256 of bf16 2 to 3 % less; but 512 workgroups 26.9 -> 30.5, 1600 of 90 tokens 24 -> 36.
        const int units = a.batch * a.c.kv_heads * a.head_groups;
        constexpr int MORE = DP == 256 ? kWaves : 2 * kWaves;
        if (units <= kGrid) k_prefix_short<E, DP, FULL, MORE><<<units, 64 * MORE, 0, st>>>(p);
        else k_prefix_short<E, DP, FULL, kWaves><<<units, 64 * kWaves, 0, st>>>(p);
        return hipGetLastError();
    }
    const Sizes z = sizes_of(a.c, a.batch, a.heads, p.groups);
    const int threads = std::max(256, (a.batch + 63) / 64 * 64);
    const int64_t pieces = z.query_bytes / 16;
    k_prefix_plan<E, DP><<<(int)(1 + (pieces + threads - 1) / threads), threads, 0, st>>>(p, z, kColumns<E, DP>);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    k_prefix<E, DP, FULL><<<kGrid, 64 * kTaskWaves<DP>, 0, st>>>(p, z);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    k_prefix_join<E><<<dim3(a.batch * a.heads, (a.c.head_dim + 127) / 128), 256, 0, st>>>(p, z, kColumns<E, DP>);
    return hipGetLastError();
}

template <typename E> hipError_t run(const PrefixArgs &p, bool few, hipStream_t st) {
    const int D = p.a.c.head_dim;
    if (D <= 64) return D == 64 ? run<E, 64, true>(p, few, st) : run<E, 64, false>(p, few, st);
    if (D <= 128) return D == 128 ? run<E, 128, true>(p, few, st) : run<E, 128, false>(p, few, st);
    return D == 256 ? run<E, 256, true>(p, few, st) : run<E, 256, false>(p, few, st);
}

}  // namespace

// A window may make a call short: the workspace goes by the table alone.
int64_t prefix_workspace(const CacheArgs &c, int batch, int heads, int groups, int width) {
    if (is_short(c, batch, heads, (int64_t)width * c.page_size)) return 0;
    return space_of(nullptr, sizes_of(c, batch, heads, groups), batch, c.head_dim).bytes;
}

hipError_t launch_prefix(const PrefixArgs &args, hipStream_t st) {
    PrefixArgs p = args;
    AttnArgs &a = p.a;
    a.head_groups = (a.group + 15) / 16, a.shares = 0;
    int64_t tokens = (int64_t)a.width * a.c.page_size;
    if (a.window) tokens = std::min<int64_t>(tokens, a.window);
    const bool few = is_short(a.c, a.batch, a.heads, tokens);
    return a.c.dtype == BSP_F32 ? run<float>(p, few, st) : run<uint16_t>(p, few, st);
}

}  // namespace bsp
