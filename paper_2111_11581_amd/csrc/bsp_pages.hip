// Care of a paged cache: fork, extend, release, compact, copy.  Tables, lengths and reference counts
// are read and changed on the device only; counts change by integer atomics, whose order does not
// matter, and pages are given out by rank, so results do not depend on scheduling.
#include <hip/hip_runtime.h>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"

namespace bsp {

namespace {

__device__ __forceinline__ bool in(int i, int n) { return (unsigned)i < (unsigned)n; }

// A pair's column of the table, or (column `width`) its length, is read, and counted, before any child's
// is changed: a workgroup owns 16 columns of all pairs, 64 pairs at a time.  A thread keeps what it
// read of its first pairs in registers and of more in scratch, which nobody else touches.  Bound by
// the latency of pair, entry and count one after the other: 32 pairs of 54 entries 3.2 us, an empty
// kernel 3 (64 columns and 4 pairs at a time, all through scratch: 14 us).
constexpr int kForkCols = 16, kForkRows = 64, kForkKept = 4;
__global__ __launch_bounds__(kForkCols *kForkRows) void k_fork(PagesArgs a, const int32_t *__restrict__ parents,
                                                               const int32_t *__restrict__ children) {
    const int col = blockIdx.x * kForkCols + threadIdx.x % kForkCols, first = threadIdx.x / kForkCols;
    const int64_t line = (int64_t)a.width + 1;
    const bool on = col <= a.width;
    int kept[kForkKept], child[kForkKept];
    auto read = [&](int i, int *to) {   // the child, or -1
        const int p = parents[i], c = children[i];
        if (!on || !in(p, a.seqs) || !in(c, a.seqs)) return -1;
        *to = col < a.width ? a.table[(int64_t)p * a.width + col] : a.lens[p];
        if (col < a.width && in(*to, a.pages)) atomicAdd(&a.refs[*to], 1);
        return c;
    };
    auto write = [&](int c, int v) {
        if (c < 0) return;
        if (col == a.width) {
            a.lens[c] = v;
            return;
        }
        const int old = atomicExch(&a.table[(int64_t)c * a.width + col], v);
        if (in(old, a.pages)) atomicSub(&a.refs[old], 1);
    };
#pragma unroll
    for (int k = 0; k < kForkKept; ++k) child[k] = first + k * kForkRows < a.n ? read(first + k * kForkRows, &kept[k]) : -1;
    for (int i = first + kForkKept * kForkRows; i < a.n; i += kForkRows) {
        int v;
        if (read(i, &v) >= 0) a.scratch[i * line + col] = v;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kForkKept; ++k) write(child[k], kept[k]);
    for (int i = first + kForkKept * kForkRows; i < a.n; i += kForkRows)
        if (on && in(parents[i], a.seqs) && in(children[i], a.seqs)) write(children[i], a.scratch[i * line + col]);
}

__global__ __launch_bounds__(256) void k_release(PagesArgs a, const int32_t *__restrict__ rows) {
    const int r = rows[blockIdx.x];
    if (!in(r, a.seqs)) return;
    for (int col = threadIdx.x; col < a.width; col += 256) {
        const int old = atomicExch(&a.table[(int64_t)r * a.width + col], -1);
        if (in(old, a.pages)) atomicSub(&a.refs[old], 1);
    }
    if (threadIdx.x == 0) a.lens[r] = 0;
}

constexpr int kScan = 1024;

// Exclusive sum over the workgroup of one value a thread, and the whole sum.
template <typename T> __device__ __forceinline__ T scan(T v, T *total) {
    __shared__ T part[kScan / 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    T sum = v;
    for (int d = 1; d < 64; d *= 2) {
        const T o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    __syncthreads();   // part may still be read by the call before
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    T before = 0, all = 0;
    for (int w = 0; w < kScan / 64; ++w) {
        if (w < wave) before += part[w];
        all += part[w];
    }
    *total = all;
    return before + sum - v;
}

// Writes the pages of [from, to) that are in use (live) or free in order, as many as `most`; returns
// how many there are, counted no further than needed.
__device__ int list_pages(const int32_t *refs, int from, int to, bool live, int32_t *list, int most) {
    int count = 0;
    for (int64_t base = from; base < to && count < most; base += kScan * 4) {
        const int64_t p = base + threadIdx.x * 4;
        int flag[4], mine = 0, total;
        for (int i = 0; i < 4; ++i) {
            flag[i] = p + i < to && (refs[p + i] > 0) == live;
            mine += flag[i];
        }
        int rank = count + scan(mine, &total);
        for (int i = 0; i < 4; ++i)
            if (flag[i]) {
                if (rank < most && list) list[rank] = (int)(p + i);
                ++rank;
            }
        count += total;
    }
    return count;
}

// What a sequence of k_extend needs: pages for its entries start .. end - 1, and one for its last
// entry `last` where that has tokens and is shared (or names no page).
struct Need {
    int have, more, last, start, end, old, fresh_last, need;
};
__device__ __forceinline__ Need need_of(const PagesArgs &a, int page_size, int row, int more) {
    Need n = {};
    n.old = -1;
    if (!in(row, a.seqs)) return n;
    n.have = max(a.lens[row], 0), n.more = max(more, 0);
    n.last = n.have / page_size;
    n.start = (int)(((int64_t)n.have + page_size - 1) / page_size);
    n.end = (int)min(((int64_t)n.have + n.more + page_size - 1) / page_size, (int64_t)INT32_MAX);   // past any width
    if (n.more == 0) return n;
    if (n.have % page_size && n.last < a.width) {
        n.old = a.table[(int64_t)row * a.width + n.last];
        if (!in(n.old, a.pages)) n.old = -1;
        n.fresh_last = n.old < 0 || a.refs[n.old] > 1;
    }
    n.need = n.end - n.start + n.fresh_last;
    return n;
}

// One workgroup, since a sequence's pages depend on what all before it take and the whole call on all:
// what every sequence needs and its rank among all, the lowest free pages, then the
// new entries.  Bound by the latency of about ten dependent accesses and barriers: 32 sequences, 612
// pages 7 us.  scratch: first rank [n], copies {src, dst} [n], free pages [pages].
__global__ __launch_bounds__(kScan) void k_extend(PagesArgs a, int page_size, const int32_t *__restrict__ rows,
                                                  const int32_t *__restrict__ counts, int32_t *__restrict__ pos) {
    __shared__ int bad;
    __shared__ Need s_need[kScan];    // of the first sequences; of more they are worked out again
    int32_t *first = a.scratch, *copy = first + a.n, *list = copy + 2 * (int64_t)a.n;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    int64_t sum = 0;
    for (int base = 0; base < a.n; base += kScan) {
        const int i = base + threadIdx.x;
        int64_t need = 0, total;
        if (i < a.n) {
            const Need n = need_of(a, page_size, rows[i], counts[i]);
            if (base == 0) s_need[i] = n;
            if (n.more && n.end > a.width) bad = 1;
            need = n.need;
        }
        const int64_t rank = scan(need, &total);
        if (i < a.n) first[i] = (int)min(sum + rank, (int64_t)INT32_MAX);
        sum += total;
    }
    __syncthreads();
    const int want = (int)min(sum, (int64_t)a.pages + 1);
    const bool ok = !bad && list_pages(a.refs, 0, a.pages, false, list, min(want, a.pages)) >= want;
    __syncthreads();
    // a wave per sequence
    for (int i = threadIdx.x / 64; i < a.n; i += kScan / 64) {
        const int row = rows[i], lane = threadIdx.x % 64;
        const Need n = i < kScan ? s_need[i] : need_of(a, page_size, row, counts[i]);
        if (lane == 0) {
            pos[i] = ok && in(row, a.seqs) ? n.have : -1;
            copy[2 * i] = ok && n.fresh_last ? n.old : -1;
            copy[2 * i + 1] = ok && n.fresh_last ? list[first[i]] : -1;
        }
        if (!ok || !n.more) continue;
        for (int e = n.start + lane; e < n.end; e += 64) {
            const int p = list[first[i] + n.fresh_last + e - n.start];
            a.table[(int64_t)row * a.width + e] = p;
            a.refs[p] = 1;
        }
    }
    __syncthreads();
    // the shared pages' entries and counts last: what a sequence needs goes by them
    if (ok)
        for (int i = threadIdx.x; i < a.n; i += kScan) {
            const int row = rows[i], more = max(counts[i], 0);
            if (!in(row, a.seqs)) continue;
            const int have = max(a.lens[row], 0), old = copy[2 * i], fresh = copy[2 * i + 1];
            if (fresh >= 0) {
                a.table[(int64_t)row * a.width + have / page_size] = fresh;
                a.refs[fresh] = 1;
                if (old >= 0) atomicSub(&a.refs[old], 1);
            }
            a.lens[row] = have + more;
        }
}

// A page is copied in chunks of 2048 pieces of 16 bytes, a workgroup per chunk: all of a thread's eight
// loads are on their way before its first store (one at a time: 12 layers' shared last pages 12 us
// instead of 6, 8 layers' compaction 136 instead of 101).  where(i) is piece i's place on both sides.
// ONCE: pages that are not read again soon go past the caches (compaction 100 -> 95 us); those that
// k_extend has replaced are shared by several children, and read next.
constexpr int kChunk = 8 * 256;
template <bool ONCE, typename F> __device__ __forceinline__ void copy_chunk(u32x4 *dst, const u32x4 *src, int from, int n, F where) {
    u32x4 v[8];
    int64_t at[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) at[k] = where(min(from + k * 256 + (int)threadIdx.x, n - 1));
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = ONCE ? __builtin_nontemporal_load(&src[at[k]]) : src[at[k]];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (from + k * 256 + (int)threadIdx.x >= n) continue;
        if (ONCE)
            __builtin_nontemporal_store(v[k], &dst[at[k]]);
        else
            dst[at[k]] = v[k];
    }
}

// The slots in use of the pages that k_extend has replaced: x the sequence, y planes, z chunks.
__global__ __launch_bounds__(256) void k_extend_copy(PagesArgs a, PlanesArgs d, int esize, const int32_t *__restrict__ pos) {
    const int i = blockIdx.x, src = a.scratch[a.n + 2 * i], dst = a.scratch[a.n + 2 * i + 1];
    if (src < 0) return;
    const int64_t unit = 16 / esize;
    // pieces of a head's slots in use, and of a head (slots first: one run of all heads)
    const int run = pos[i] % d.c.page_size * (int)(d.c.slot_stride / unit);
    const int n = run * (d.c.order == BSP_SLOT_MAJOR ? 1 : d.c.kv_heads), head = (int)(d.c.head_stride / unit);
    for (int plane = blockIdx.y; plane < d.planes; plane += gridDim.y) {
        u32x4 *base = (u32x4 *)d.data + plane * (d.plane_stride / unit);
        for (int from = blockIdx.z * kChunk; from < n; from += gridDim.z * kChunk)
            copy_chunk<false>(base + dst * (d.c.page_stride / unit), base + src * (d.c.page_stride / unit), from, n, [&](int k) {
                const int h = k / run;
                return (int64_t)h * head + (k - h * run);
            });
    }
}

// One workgroup: pages in use, the moves, counts and the page that each becomes; three passes over the
// counts, 4096 pages at a time, 6.6 us for the smallest caches.  scratch: moves, src [pages], dst
// [pages], map [pages].
__global__ __launch_bounds__(kScan) void k_compact_plan(PagesArgs a, int32_t *__restrict__ info) {
    int32_t *src = a.scratch + 4, *dst = src + a.pages, *map = dst + a.pages;
    const int used = list_pages(a.refs, 0, a.pages, true, nullptr, INT32_MAX);
    const int moves = list_pages(a.refs, used, a.pages, true, src, INT32_MAX);
    list_pages(a.refs, 0, used, false, dst, INT32_MAX);
    for (int64_t p = threadIdx.x; p < a.pages; p += kScan) map[p] = (int)p;
    __syncthreads();
    for (int i = threadIdx.x; i < moves; i += kScan) {
        map[src[i]] = dst[i];
        a.refs[dst[i]] = a.refs[src[i]];
        a.refs[src[i]] = 0;
    }
    if (threadIdx.x == 0) {
        a.scratch[0] = moves;
        info[0] = used, info[1] = moves;
    }
}

// Pieces of 16 bytes in a page.
__host__ __device__ __forceinline__ int pieces(const PlanesArgs &d, int esize) {
    return (int)((int64_t)d.c.page_size * d.c.kv_heads * d.c.head_dim * esize / 16);
}

// Whole pages: `n` pairs, or (compact) as many as scratch says, whose table entries follow them.  Bound
// by memory: 470 MB read and written in 93 to 100 us, 4.7 to 5 TB/s, as a large copy.
__global__ __launch_bounds__(256) void k_page_copy(PagesArgs a, PlanesArgs d, int esize, const int32_t *__restrict__ src,
                                                   const int32_t *__restrict__ dst) {
    int n = a.n;
    if (a.scratch) {
        n = a.scratch[0];
        const int32_t *map = a.scratch + 4 + 2 * (int64_t)a.pages;
        for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)a.seqs * a.width; i += gridDim.x * 256ll) {
            const int p = a.table[i];
            if (in(p, a.pages)) a.table[i] = map[p];
        }
    }
    const int64_t unit = 16 / esize;
    const int size = pieces(d, esize), chunks = (size + kChunk - 1) / kChunk;
    const int64_t per = (int64_t)d.planes * chunks;
    for (int64_t i = blockIdx.x; i < n * per; i += gridDim.x) {
        const int pair = (int)(i / per), rest = (int)(i - pair * per), plane = rest / chunks;
        const int s = src[pair], t = dst[pair];
        if (!in(s, d.c.pages) || !in(t, d.c.pages)) continue;
        u32x4 *base = (u32x4 *)d.data + plane * (d.plane_stride / unit);
        copy_chunk<true>(base + t * (d.c.page_stride / unit), base + s * (d.c.page_stride / unit), (rest - plane * chunks) * kChunk,
                   size, [](int k) { return k; });
    }
}

int esize(const PlanesArgs &d) { return d.c.dtype == BSP_F32 ? 4 : 2; }
unsigned copy_grid(int64_t items) { return (unsigned)std::min<int64_t>(std::max<int64_t>(items, 1), 256 * 8); }

}  // namespace

// fork: n lines of width + 1; extend: 3 n + pages; compact: 4 + 3 pages
int64_t pages_scratch(int pages, int width, int n) {
    return 4 * std::max({(int64_t)n * ((int64_t)width + 1), 3 * (int64_t)n + pages, 4 + 3 * (int64_t)pages});
}

hipError_t launch_fork(const PagesArgs &a, const int32_t *parents, const int32_t *children, hipStream_t st) {
    k_fork<<<(unsigned)(a.width / kForkCols + 1), kForkCols * kForkRows, 0, st>>>(a, parents, children);
    return hipGetLastError();
}

hipError_t launch_release(const PagesArgs &a, const int32_t *rows, hipStream_t st) {
    k_release<<<a.n, 256, 0, st>>>(a, rows);
    return hipGetLastError();
}

hipError_t launch_extend(const PagesArgs &a, const PlanesArgs &d, const int32_t *rows, const int32_t *counts, int32_t *pos,
                         hipStream_t st) {
    k_extend<<<1, kScan, 0, st>>>(a, d.c.page_size, rows, counts, pos);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || d.planes == 0) return e;
    const int chunks = std::min(div_up(pieces(d, esize(d)), kChunk), 64);
    k_extend_copy<<<dim3(a.n, std::min(d.planes, 65535), chunks), 256, 0, st>>>(a, d, esize(d), pos);
    return hipGetLastError();
}

hipError_t launch_compact(const PagesArgs &a, const PlanesArgs &d, int32_t *info, hipStream_t st) {
    k_compact_plan<<<1, kScan, 0, st>>>(a, info);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int32_t *src = a.scratch + 4;
    const int64_t items = std::max((int64_t)a.pages / 2 * d.planes * div_up(pieces(d, esize(d)), kChunk), div_up64((int64_t)a.seqs * a.width, 256));
    k_page_copy<<<copy_grid(items), 256, 0, st>>>(a, d, esize(d), src, src + a.pages);
    return hipGetLastError();
}

hipError_t launch_page_copy(const PlanesArgs &d, int n, const int32_t *src, const int32_t *dst, hipStream_t st) {
    PagesArgs a = {};
    a.n = n;
    k_page_copy<<<copy_grid((int64_t)n * d.planes * div_up(pieces(d, esize(d)), kChunk)), 256, 0, st>>>(a, d, esize(d), src, dst);
    return hipGetLastError();
}

}  // namespace bsp
