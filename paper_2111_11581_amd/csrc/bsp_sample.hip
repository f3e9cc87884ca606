// The next token of rows of logits: temperature, top-k, top-p and min-p, by given random numbers.
//
// What is kept is always the first of the tokens in order (falling logit, rising index), so that it is
// told by a logit and by how many of the tokens that have just it are kept.  Both are found without a sort, by
// counting and by adding up whole numbers, which has no order that could show: tokens fall into bins by
// their logit's distance from the largest, and the bin in which a cut falls is cut further by the bits of
// its keys.
//  * Rows of up to 32768 tokens stay in the LDS of a workgroup (k_sample_row), where each step waits for the one
//    before: one row of 4000 tokens takes 7.4 us without a cut and 16.6 with three, 64 rows 20.3, 64 rows of 30000 36.5.
//  * Of longer ones k_sample_scan finds the largest logits, k_sample_bins fills the bins of each chunk, and in
//    k_sample_pick a workgroup a row finds cuts and token; it reads again the tokens of the bins where the cuts
//    are, and one chunk.
//  * Rows whose elements lie apart are laid out by k_sample_lay.
// 64 rows of 131072 tokens, three cuts, 33.5 MB, 64 us in a graph: 16 laid out (67 MB, 4.2 TB/s), 25 for the bins (19
// without cuts; neither weights nor atomics bound them, but four workgroups a CU that wait in step), 25 for cuts and
// tokens (a chain of latencies, the more the more cuts).
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"

namespace bsp {

namespace {

constexpr double kOne = 8796093022208.0;   // 2^43: what a weight of 1 counts; 2^20 of them add up to 2^63, which unsigned sums hold
constexpr int kBins = 512, kSpan = 32;    // bins, and the distance that they cover: e^-32 is below 2^-44
constexpr int kScan = 2048, kLay = 256;    // tokens whose largest logit k_sample_scan and k_sample_lay find
constexpr int kChunk = 8192;               // tokens whose bins k_sample_bins fills
// Tokens that a workgroup holds in LDS.  Chunks would give more workgroups to few rows, but in three kernels: 12000 tokens
// 21.9 us and in chunks 30.9, 16 rows of them 24.5 and 33.5, 30000 tokens 30.3 and 32.2, 64 rows of them 36 and 45.
constexpr int kRow = 32768;
// Tokens of a bin that are compared with each other, a thread a token, each with all others; 32 take the same time at
// every size tried.
constexpr int kQuick = 128;
constexpr int kList = 4096;                // tokens of a bin that k_sample_pick holds in LDS
// Tokens of a chunk's first bins that k_sample_bins lists: enough for most cuts, which are among the likeliest tokens
// (64 rows of 131072 tokens 64.0 us, with 512 67.5).
constexpr int kFirst = 256;

// Logits as numbers that are in the same order; NaN and -Inf, which are never taken, are 0.
__device__ __forceinline__ uint32_t key_of(float l) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t u = __float_as_uint(l + 0.f);   // -0 as 0
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t key_of(uint16_t l) { return key_of(bf16_to_f32(l)); }
__device__ __forceinline__ uint32_t key_of(uint32_t key) { return key; }   // laid out by k_sample_lay
__device__ __forceinline__ float logit_of(uint32_t key) {
    return key == 0 ? -INFINITY : __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}

typedef __attribute__((ext_vector_type(4))) uint16_t u16x4;

// What a row is sampled with, read before anything waits.
struct Setting {
    float t, top_p, min_p, u;
    int top_k;
    __device__ __forceinline__ Setting(const SampleArgs &a, int b) {
        t = a.temperature ? a.temperature[b] : 1.f, top_k = a.top_k ? a.top_k[b] : 0;
        top_p = a.top_p ? a.top_p[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f, u = a.u[b];
    }
};

struct Row {
    uint32_t top_key;
    float top, t;        // the largest logit, the temperature
    double steps;        // 64 / (temperature ln 2)
    float bins;          // of a distance of 1
    bool greedy;
    const double *powers;   // 2^(i / 64)

    __device__ __forceinline__ Row(float temperature, uint32_t key, const double *p) : top_key(key), t(temperature), powers(p) {
        greedy = !(t > 0.f);
        top = logit_of(key), steps = 92.332482616893656877 / t, bins = (float)((double)(kBins / kSpan) / t);
    }
    // The weight in units of 2^-43.  2^(x / 64) for x = i + f, |f| <= 1/2, is 2^(i / 64) (1 + ... + (f ln 2 / 64)^5 / 120),
    // to 2^-53; adding 2^52 rounds to a whole number, to the nearest, ties to even.
    __device__ __forceinline__ uint64_t mass(uint32_t key) const {
        if (key == top_key) return (uint64_t)kOne;
        const double x = ((double)logit_of(key) - (double)top) * steps;
        if (!(x > -64.0 * 46)) return 0;   // also where the largest is Inf, or the key that of no token
        const double whole = rint(x), r = (x - whole) * 0.010830424696249145;
        double p = __builtin_fma(r, 1.0 / 120, 1.0 / 24);
        p = __builtin_fma(p, r, 1.0 / 6), p = __builtin_fma(p, r, 0.5), p = __builtin_fma(p, r, 1.0), p = __builtin_fma(p, r, 1.0);
        const int i = (int)whole;
        const double w = __builtin_ldexp(p * powers[i & 63], 43 + (i >> 6));
        return __builtin_bit_cast(uint64_t, w + 0x1p52) - __builtin_bit_cast(uint64_t, 0x1p52);
    }
    // Whether the weight is at least min_p.
    __device__ __forceinline__ bool reaches(uint32_t key, float min_p) const {
        if (key == top_key) return true;
        if (top == INFINITY) return !(0.f < min_p);
        return !(exp(((double)logit_of(key) - (double)top) * (steps * 0.010830424696249145)) < min_p);
    }
    // Never less for a smaller logit, as each rounding keeps the order.
    __device__ __forceinline__ int bin(uint32_t key) const {
        if (key == top_key) return 0;
        const float x = (top - logit_of(key)) * bins;
        return x < (float)(kBins - 1) ? (int)x : kBins - 1;   // not a number (Inf * 0): the last
    }
};
constexpr uint32_t kLeast = 0x00800000u;   // key of the smallest number

template <int THREADS> struct Scratch {
    static constexpr int WAVES = THREADS / 64;
    uint64_t mass[2][kBins];   // of bins, and of the pieces into which one is cut
    double powers[64];
    uint64_t part[2][WAVES], found[4], list_mass[kQuick];
    uint32_t count[2][kBins], key[WAVES], list_key[kQuick], listed;
    int list_index[kQuick];
};

// Inclusive scans of two values over the workgroup.
template <int THREADS> __device__ __forceinline__ void scan(uint64_t *x, uint64_t *y, uint64_t (*s_part)[THREADS / 64]) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    *x = wave_scan(*x, Sum()), *y = wave_scan(*y, Sum());
    __syncthreads();
    if (lane == 63) s_part[0][wave] = *x, s_part[1][wave] = *y;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w)
        if (w < wave) *x += s_part[0][w], *y += s_part[1][w];
}
// Largest over the workgroup, for all.
template <int THREADS> __device__ __forceinline__ uint32_t largest(uint32_t v, uint32_t *s_part) {
    v = wave_all(v, Largest());
    __syncthreads();
    if (threadIdx.x % 64 == 0) s_part[threadIdx.x / 64] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v = max(v, s_part[w]);
    return v;
}

template <int THREADS> __device__ __forceinline__ void start(Scratch<THREADS> &s) {
    if (threadIdx.x < 64) s.powers[threadIdx.x] = exp2(threadIdx.x / 64.0);
}
template <int THREADS> __device__ __forceinline__ void clear(Scratch<THREADS> &s, int which) {
    for (int i = threadIdx.x; i < kBins; i += THREADS) s.count[which][i] = 0, s.mass[which][i] = 0;
}
template <int THREADS> __device__ __forceinline__ void add(Scratch<THREADS> &s, int which, int bin, uint64_t mass) {
    atomicAdd(&s.count[which][bin], 1u);
    if (mass) atomicAdd((unsigned long long *)&s.mass[which][bin], (unsigned long long)mass);
}

// The first bin up to which `target` tokens, or that much mass, come together; there is one.
struct Found {
    int bin;
    uint64_t count_before, mass_before, count;
};
template <int THREADS> __device__ __forceinline__ Found locate(Scratch<THREADS> &s, int which, bool by_mass, uint64_t target) {
    constexpr int PER = kBins / THREADS < 1 ? 1 : kBins / THREADS;
    const int t = threadIdx.x;
    uint64_t count = 0, mass = 0;
    if (t * PER < kBins)
#pragma unroll
        for (int i = 0; i < PER; ++i) count += s.count[which][t * PER + i], mass += s.mass[which][t * PER + i];
    uint64_t counts = count, masses = mass;
    scan<THREADS>(&counts, &masses, s.part);
    const uint64_t upto = by_mass ? masses : counts, before = upto - (by_mass ? mass : count);
    if (before < target && target <= upto) {
        counts -= count, masses -= mass;
        int i = t * PER;
        for (; i < t * PER + PER - 1; ++i) {
            if ((by_mass ? masses + s.mass[which][i] : counts + s.count[which][i]) >= target) break;
            counts += s.count[which][i], masses += s.mass[which][i];
        }
        s.found[0] = i, s.found[1] = counts, s.found[2] = masses, s.found[3] = s.count[which][i];
    }
    __syncthreads();
    const Found f = {(int)s.found[0], s.found[1], s.found[2], s.found[3]};
    __syncthreads();
    return f;
}

// Of the keys lo .. hi that each(f) calls f with, in any order, the one down to which `target` of them, or that much of
// mass(key), come together; nine bits at a time.  `count`: how many have it.
template <int THREADS, typename F, typename M>
__device__ __forceinline__ Found select(Scratch<THREADS> &s, uint32_t lo, uint32_t hi, bool by_mass, uint64_t target, F each, M mass,
                                        uint32_t *key) {
    uint64_t counts = 0, masses = 0;
    for (;;) {
        const int shift = max(0, 32 - (hi == lo ? 32 : __clz((int)(hi - lo))) - 9);
        clear(s, 1);
        __syncthreads();
        each([&](uint32_t k) {
            if (k >= lo && k <= hi) add(s, 1, (int)((hi - k) >> shift), mass(k));
        });
        __syncthreads();
        Found f = locate(s, 1, by_mass, target);
        target -= by_mass ? f.mass_before : f.count_before;
        counts += f.count_before, masses += f.mass_before;
        const uint32_t top = hi - ((uint32_t)f.bin << shift);
        if (shift == 0) {
            *key = top;
            f.count_before = counts, f.mass_before = masses;
            return f;
        }
        lo = max((int64_t)lo, (int64_t)top - ((1ll << shift) - 1)), hi = top;
    }
}

// The first key of lo .. hi for which `holds`, which does for all above and for hi: by a wave, 64 places at a time.
template <typename P> __device__ __forceinline__ uint32_t first_key(uint32_t lo, uint32_t hi, P holds) {
    while (lo < hi) {
        const uint32_t step = (hi - lo - 1) / 64 + 1;
        const uint64_t at = lo + (uint64_t)(threadIdx.x % 64) * step;
        const uint64_t hit = __ballot(at >= hi || holds((uint32_t)at));
        const int first = hit ? __ffsll((unsigned long long)hit) - 1 : 64;   // of 64 places
        hi = (uint32_t)min((uint64_t)hi, lo + (uint64_t)first * step);
        if (first) lo += (first - 1) * step + 1;
    }
    return hi;
}

// The first key whose weight is at least min_p: beside where its logarithm says, or else wherever it is.
__device__ __forceinline__ uint32_t least_key(const Row &row, float min_p) {
    auto holds = [&](uint32_t k) { return row.reaches(k, min_p); };
    const uint32_t guess = min(key_of((float)((double)row.top + log((double)min_p) * (double)row.t)), row.top_key);
    const uint32_t lo = guess > kLeast + 32 ? guess - 32 : kLeast;
    const uint64_t hit = __ballot(holds(min(lo + threadIdx.x % 64, row.top_key)));
    const int first = hit ? __ffsll((unsigned long long)hit) - 1 : 64;
    if (first == 0 && lo > kLeast) return first_key(kLeast, lo, holds);
    return first < 64 ? min(lo + first, row.top_key) : first_key(lo + 64, row.top_key, holds);
}

// What is kept of a row: tokens whose key is above, and of those that have it the ones up to an index.
struct Kept {
    uint32_t key, index;
    __device__ __forceinline__ bool has(uint32_t k, int i) const { return k > key || (k == key && (uint32_t)i <= index); }
};

// Cuts what is kept of a row, in a bin of `in.count` tokens, where `target` of its tokens, or that much mass, come together;
// returns their number and mass in `in`.  prepare(bin, count) is told the bin and how many tokens it has, and
// each_token(f) calls f(key, index) for these at least.
//  * Few tokens are compared with each other, a thread for each.
//  * Of more the key is found by its bits, and where several tokens have it the last index in the same way.
template <int THREADS, typename R, typename T>
__device__ __forceinline__ void cut_bin(Scratch<THREADS> &s, const Row &row, Found *in, bool by_mass, uint64_t target, R prepare, T each_token,
                                        Kept *kept) {
    prepare(in->bin, in->count);
    const Kept from = *kept;
    if (in->count <= kQuick) {
        const int t = threadIdx.x;
        if (t == 0) s.listed = 0;
        __syncthreads();
        each_token([&](uint32_t k, int i) {
            if (!from.has(k, i) || row.bin(k) != in->bin) return;
            const uint32_t at = atomicAdd(&s.listed, 1u);
            if (at < kQuick) s.list_key[at] = k, s.list_index[at] = i, s.list_mass[at] = row.mass(k);
        });
        __syncthreads();
        const int n = min((int)s.listed, kQuick);
        if (t < n) {
            const uint32_t k = s.list_key[t];
            const int i = s.list_index[t];
            uint64_t mass = 0, count = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const uint32_t o = s.list_key[j];
                const bool before = o > k || (o == k && s.list_index[j] <= i);
                count += before, mass += before ? s.list_mass[j] : 0;
            }
            const uint64_t upto = by_mass ? mass : count, own = by_mass ? s.list_mass[t] : 1;
            if (upto >= target && upto - own < target) s.found[0] = k, s.found[1] = i, s.found[2] = count, s.found[3] = mass;
        }
        __syncthreads();
        kept->key = (uint32_t)s.found[0], kept->index = (uint32_t)s.found[1], in->count = s.found[2], in->mass_before += s.found[3];
        return;
    }
    const uint32_t hi = in->bin == 0 ? row.top_key : first_key(kLeast, row.top_key, [&](uint32_t k) { return row.bin(k) < in->bin; }) - 1;
    const uint32_t lo = in->bin == kBins - 1 ? kLeast : first_key(kLeast, row.top_key, [&](uint32_t k) { return row.bin(k) <= in->bin; });
    uint32_t key;
    const Found at = select(s, max(lo, from.key), hi, by_mass, target, [&](auto f) {
        each_token([&](uint32_t k, int i) { if (from.has(k, i)) f(k); });
    }, [&](uint32_t k) { return row.mass(k); }, &key);
    const uint64_t one = row.mass(key), rest = target - (by_mass ? at.mass_before : at.count_before);
    const uint64_t equal = by_mass ? (rest + one - 1) / one : rest;
    in->mass_before += at.mass_before + equal * one;
    kept->key = key, kept->index = key == from.key ? from.index : 0xffffffffu;
    if (equal < at.count) {   // the lower index first
        uint32_t from_end;
        select(s, 0, kMostVocab - 1, false, equal, [&](auto f) {
            each_token([&](uint32_t k, int i) { if (k == key && from.has(k, i)) f((uint32_t)(kMostVocab - 1 - i)); });
        }, [](uint32_t) { return (uint64_t)0; }, &from_end);
        kept->index = kMostVocab - 1 - from_end;
    }
}

// The cuts of a row of `live` tokens, whose bins hold their numbers; fill_mass(kept) adds their mass for what is kept, and
// returns all of it.
template <int THREADS, typename R, typename T, typename M>
__device__ __forceinline__ Kept cut(const Setting &set, Scratch<THREADS> &s, const Row &row, uint64_t live, R prepare, T each_token,
                                    M fill_mass) {
    const bool by_k = set.top_k > 0 && (uint64_t)set.top_k < live, by_p = set.top_p < 1.f;
    Kept kept = {kLeast, 0xffffffffu};
    Found in;
    if (by_k) {
        in = locate(s, 0, false, (uint64_t)set.top_k);
        cut_bin(s, row, &in, false, set.top_k - in.count_before, prepare, each_token, &kept);
    }
    if (by_p) {
        const uint64_t all = fill_mass(kept, by_k, in);
        const uint64_t target = max((uint64_t)1, (uint64_t)ceil(fmax((double)set.top_p, 0.0) * (double)all));
        in = locate(s, 0, true, target);   // at most the bin of the first cut, of which not all is kept
        cut_bin(s, row, &in, true, target - in.mass_before, prepare, each_token, &kept);
    }
    if (set.min_p > 0.f) {
        const uint32_t least = least_key(row, set.min_p);
        if (least > kept.key) kept = {least, 0xffffffffu};
    }
    return kept;
}

// Where among a sum the token is.
__device__ __forceinline__ uint64_t place_of(float u, uint64_t total) {
    return (uint64_t)((double)fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * (double)total);   // the sum has to be more
}
__device__ __forceinline__ void put(const SampleArgs &a, int b, int token, uint64_t mass, uint64_t total) {
    a.tokens[b] = token;
    if (a.logp) a.logp[b] = token < 0 ? -INFINITY : (float)log((double)mass / (double)total);
}

// Keys of elements i .. i + 3 of a row, 0 past its end; ALONG: elements are side by side.
template <typename E, bool ALONG> struct Source {
    const E *row;
    int64_t stride;
    int vocab;
    bool whole;   // whether four at a time begin at a multiple of their size
    __device__ __forceinline__ Source(const void *logits, int b, int64_t row_stride, int64_t token_stride, int v)
        : row((const E *)logits + b * row_stride), stride(token_stride), vocab(v), whole(ALONG && (uintptr_t)row % (4 * sizeof(E)) == 0) {}
    __device__ __forceinline__ uint32_t one(int i) const { return i < vocab ? key_of(row[ALONG ? i : i * stride]) : 0; }
    __device__ __forceinline__ void four(int i, uint32_t *key) const {
        if (ALONG && whole && i + 4 <= vocab) {
            if constexpr (sizeof(E) == 4) {
                const u32x4 v = *(const u32x4 *)(row + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bits = v[e];   // a bit cast of v[e] itself takes the first element
                    key[e] = key_of(__builtin_bit_cast(E, bits));
                }
            } else {
                const u16x4 v = *(const u16x4 *)(row + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) key[e] = key_of((E)v[e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) key[e] = one(i + e);
        }
    }
};

// A workgroup for a row of up to MOST tokens, whose keys it holds in LDS, four at a time.
template <typename E, bool ALONG, int THREADS, int MOST>
__global__ __launch_bounds__(THREADS) void k_sample_row(SampleArgs a) {
    constexpr int WAVES = THREADS / 64;
    __shared__ Scratch<THREADS> s;
    __shared__ u32x4 s_key[MOST / 4];
    __shared__ uint64_t s_sum[MOST / (4 * THREADS) * WAVES];
    const int b = blockIdx.x, t = threadIdx.x, lane = t % 64, wave = t / 64;
    const Source<E, ALONG> src(a.logits, b, a.row_stride, a.token_stride, a.vocab);
    const Setting set(a, b);
    const int fours = (a.vocab + 3) / 4, rounds = (fours + THREADS - 1) / THREADS;
    uint32_t top = 0;
#pragma unroll 4
    for (int i = t; i < rounds * THREADS; i += THREADS) {
        uint32_t key[4];
        src.four(4 * i, key);
        s_key[i] = (u32x4){key[0], key[1], key[2], key[3]};
        top = max(max(top, max(key[0], key[1])), max(key[2], key[3]));
    }
    start(s);
    top = largest<THREADS>(top, s.key);
    if (top == 0) {
        if (t == 0) put(a, b, -1, 0, 0);
        return;
    }
    const Row row(set.t, top, s.powers);
    auto each_token = [&](auto f) {   // of the thread's own
#pragma unroll 1
        for (int i = t; i < fours; i += THREADS) {
            const u32x4 k = s_key[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) f(k[e], 4 * i + e);
        }
    };
    if (row.greedy) {
        uint32_t from_end = 0;
        each_token([&](uint32_t k, int i) { if (k == top) from_end = max(from_end, (uint32_t)(kMostVocab - i)); });
        from_end = largest<THREADS>(from_end, s.key);
        if (t == 0) put(a, b, kMostVocab - from_end, 1, 1);
        return;
    }
    Kept kept = {kLeast, 0xffffffffu};
    if (a.top_k || a.top_p || a.min_p) {
        const bool by_count = set.top_k > 0;
        clear(s, 0);
        __syncthreads();
        uint64_t live = 0, all = 0;
        if (by_count) {
            each_token([&](uint32_t k, int) {
                if (k) ++live, atomicAdd(&s.count[0][row.bin(k)], 1u);
            });
            scan<THREADS>(&live, &all, s.part);
            if (t == THREADS - 1) s.found[0] = live;
            __syncthreads();
            live = s.found[0];
        }
        kept = cut(set, s, row, live, [](int, uint64_t) {}, each_token, [&](const Kept &k0, bool, const Found &) {
            if (by_count) clear(s, 0);   // bins of what is kept alone
            __syncthreads();
            uint64_t all = 0, none = 0;
            each_token([&](uint32_t k, int i) {
                if (!k0.has(k, i)) return;
                const uint64_t m = row.mass(k);
                add(s, 0, row.bin(k), m), all += m;
            });
            scan<THREADS>(&all, &none, s.part);
            if (t == THREADS - 1) s.found[0] = all;
            __syncthreads();
            all = s.found[0];
            return all;
        });
    }
    auto mass = [&](uint32_t k, int i) { return kept.has(k, i) ? row.mass(k) : 0; };
#pragma unroll 1
    for (int q = 0; q < rounds; ++q) {
        const u32x4 k = s_key[q * THREADS + t];
        uint64_t m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) m += mass(k[e], 4 * (q * THREADS + t) + e);
        if (__any(m != 0)) m = wave_all(m, Sum());
        if (lane == 0) s_sum[q * WAVES + wave] = m;
    }
    __syncthreads();
    // by each wave for itself: where among these sums the token is
    const int sums = rounds * WAVES;
    uint64_t total = 0;
    for (int i = lane; i < sums; i += 64) total += s_sum[i];
    total = wave_all(total, Sum());
    const uint64_t target = place_of(set.u, total);
    uint64_t before = 0;
    int at = 0;
    for (int i0 = 0; i0 < sums; i0 += 64) {
        const uint64_t m = i0 + lane < sums ? s_sum[i0 + lane] : 0;
        const uint64_t upto = wave_scan(m, Sum());
        const uint64_t hit = __ballot(before + upto > target);
        if (hit) {
            const int first = __ffsll((unsigned long long)hit) - 1;
            at = i0 + first, before += of_lane(upto - m, first);
            break;
        }
        before += of_lane(upto, 63);
    }
    if (at % WAVES != wave) return;
    const int i = at / WAVES * THREADS + t;
    const u32x4 k = s_key[i];
    uint64_t m[4], upto = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) upto += m[e] = mass(k[e], 4 * i + e);
    const uint64_t mine = upto;
    upto = wave_scan(upto, Sum());
    upto += before - mine;   // before the lane's
    if (upto > target || upto + mine <= target) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (upto <= target && upto + m[e] > target) put(a, b, 4 * i + e, m[e], total);
        upto += m[e];
    }
}

// ---- longer rows -------------------------------------------------------------------------------------

struct Space {
    uint32_t *keys, *top;        // [batch][vocab] if rows are laid out; [batch][scans]
    uint32_t *count;             // [batch][chunks][bins]
    uint64_t *mass;
    int2 *listed;                // [batch][chunks]: bins whose tokens are listed, and how many these are
    uint2 *token;                // [batch][chunks][kFirst]: their keys and indexes, in any order
    int scan, scans, chunks, row;   // tokens of a scan; elements from a row of keys to the next
    int64_t bytes;
};
__host__ __device__ inline Space space_of(void *workspace, int batch, int vocab, bool apart) {
    Space s;
    char *at = (char *)workspace;
    auto take = [&](int64_t bytes) {
        char *here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    s.scan = apart ? kLay : kScan, s.scans = (vocab + s.scan - 1) / s.scan, s.chunks = vocab > kRow ? (vocab + kChunk - 1) / kChunk : 0, s.row = (vocab + 3) / 4 * 4;
    s.keys = (uint32_t *)take(apart ? (int64_t)batch * s.row * 4 : 0);
    s.top = (uint32_t *)take((int64_t)batch * s.scans * 4);
    s.mass = (uint64_t *)take((int64_t)batch * s.chunks * kBins * 8);
    s.count = (uint32_t *)take((int64_t)batch * s.chunks * kBins * 4);
    s.listed = (int2 *)take((int64_t)batch * s.chunks * 8);
    s.token = (uint2 *)take((int64_t)batch * s.chunks * kFirst * 8);
    s.bytes = at - (char *)workspace;
    return s;
}

// The largest key of 2048 elements of a row that lie side by side.
template <typename E> __global__ __launch_bounds__(256) void k_sample_scan(SampleArgs a, Space sp) {
    __shared__ uint32_t s_part[4];
    const int b = blockIdx.y, c = blockIdx.x, t = threadIdx.x;
    const Source<E, true> src(a.logits, b, a.row_stride, 1, a.vocab);
    uint32_t key[8], top = 0;
#pragma unroll
    for (int q = 0; q < 2; ++q) src.four(c * kScan + 4 * (q * 256 + t), key + 4 * q);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, key[j]);
    top = largest<256>(top, s_part);
    if (t == 0) sp.top[(int64_t)b * sp.scans + c] = top;
}
// The same for 256 tokens of 16 rows whose elements lie apart, and their keys, laid out, through LDS: read along the
// rows where they begin side by side.
template <typename E> __global__ __launch_bounds__(256) void k_sample_lay(SampleArgs a, Space sp) {
    constexpr int ROWS = 16;
    __shared__ uint32_t s_key[ROWS][kLay + 1], s_top[ROWS][4];
    const int b0 = blockIdx.y * ROWS, rows = min(ROWS, a.batch - b0), t = threadIdx.x, lane = t % 64, wave = t / 64, i0 = blockIdx.x * kLay;
    const bool along_rows = rows > 1 && a.row_stride > -a.token_stride && a.row_stride < a.token_stride;
    const int r0 = along_rows ? t % ROWS : 0, at0 = along_rows ? t / ROWS : t;         // the thread's first, and from
    const int next_r = along_rows ? 0 : 1, next_at = along_rows ? kLay / ROWS : 0;   // each to the next
    E v[ROWS];
    const E *src = (const E *)a.logits + b0 * a.row_stride + i0 * a.token_stride;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int r = min(r0 + k * next_r, rows - 1), i = min(at0 + k * next_at, a.vocab - 1 - i0);
        v[k] = src[r * a.row_stride + i * a.token_stride];
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int r = r0 + k * next_r, i = at0 + k * next_at;
        s_key[r][i] = r < rows && i0 + i < a.vocab ? key_of(v[k]) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const uint32_t k = s_key[r][t];
        if (r < rows && i0 + t < a.vocab) sp.keys[(int64_t)(b0 + r) * sp.row + i0 + t] = k;
        const uint32_t top = wave_all(k, Largest());
        if (lane == 0) s_top[r][wave] = top;
    }
    __syncthreads();
    if (t < rows) sp.top[(int64_t)(b0 + t) * sp.scans + blockIdx.x] = max(max(s_top[t][0], s_top[t][1]), max(s_top[t][2], s_top[t][3]));
}

// The largest key of a row, for all threads.
template <int THREADS> __device__ __forceinline__ uint32_t top_of(const Space &sp, int b, uint32_t *s_part) {
    uint32_t top = 0;
    for (int i = threadIdx.x; i < sp.scans; i += THREADS) top = max(top, sp.top[(int64_t)b * sp.scans + i]);
    return largest<THREADS>(top, s_part);
}

// Bins of a chunk, and the tokens of its first ones.
template <typename E> __global__ __launch_bounds__(512) void k_sample_bins(SampleArgs a, Space sp) {
    constexpr int T = 512, Q = kChunk / (4 * T);
    __shared__ Scratch<T> s;
    const int b = blockIdx.y, c = blockIdx.x, t = threadIdx.x;
    const Source<E, true> src(a.logits, b, a.row_stride, 1, a.vocab);
    const Setting set(a, b);
    uint32_t key[Q][4];
#pragma unroll
    for (int q = 0; q < Q; ++q) src.four(c * kChunk + 4 * (q * T + t), key[q]);
    start(s);
    clear(s, 0);
    if (t == 0) s.listed = 0;
    const uint32_t top = top_of<T>(sp, b, s.key);
    const Row row(set.t, top, s.powers);
    if (top == 0 || row.greedy) return;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (key[q][e]) add(s, 0, row.bin(key[q][e]), row.mass(key[q][e]));
    __syncthreads();
    const int64_t at = ((int64_t)b * sp.chunks + c) * kBins;
    for (int i = t; i < kBins; i += T) sp.count[at + i] = s.count[0][i], sp.mass[at + i] = s.mass[0][i];
    if (!a.top_k && !a.top_p && !a.min_p) return;
    // the first bins that have no more than kFirst tokens
    constexpr int PER = kBins / T;
    uint64_t count = 0, none = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) count += s.count[0][t * PER + i];
    uint64_t upto = count;
    scan<T>(&upto, &none, s.part);
    upto -= count;
    int mine = 0;   // of the thread's bins
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        upto += s.count[0][t * PER + i];
        if (upto <= kFirst) mine = t * PER + i + 1;
    }
    const int bins = (int)largest<T>((uint32_t)mine, s.key);
    uint2 *list = sp.token + ((int64_t)b * sp.chunks + c) * kFirst;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (key[q][e] && row.bin(key[q][e]) < bins)
                list[atomicAdd(&s.listed, 1u)] = make_uint2(key[q][e], (uint32_t)(c * kChunk + 4 * (q * T + t) + e));
    __syncthreads();
    if (t == 0) sp.listed[(int64_t)b * sp.chunks + c] = make_int2(bins, (int)s.listed);
}

// Cuts and token of a row.
template <typename E> __global__ __launch_bounds__(1024) void k_sample_pick(SampleArgs a, Space sp) {
    constexpr int T = 1024, WAVES = T / 64, MOST = kMostVocab / kChunk;
    __shared__ Scratch<T> s;
    __shared__ uint32_t s_key[kList], s_listed;
    __shared__ int s_index[kList], s_bins;
    __shared__ int2 s_listed_of[MOST];
    __shared__ uint64_t s_chunk[MOST];
    const int b = blockIdx.x, t = threadIdx.x, lane = t % 64, wave = t / 64;
    const Source<E, true> src(a.logits, b, a.row_stride, 1, a.vocab);
    const Setting set(a, b);
    const bool cut_at_all = a.top_k || a.top_p || a.min_p;
    const uint32_t *counts = sp.count + (int64_t)b * sp.chunks * kBins;
    const uint64_t *masses = sp.mass + (int64_t)b * sp.chunks * kBins;
    auto read_list = [&](int c, uint2 (&v)[kFirst / 64]) {   // past its end whatever is there
#pragma unroll
        for (int i = 0; i < kFirst / 64; ++i) v[i] = sp.token[((int64_t)b * sp.chunks + c) * kFirst + 64 * i + lane];
    };
    static_assert(WAVES * kFirst <= kList, "");
    bool held = cut_at_all && sp.chunks <= WAVES;   // all lists in LDS, read before anything waits
    if (held && wave < sp.chunks) {
        uint2 v[kFirst / 64];
        read_list(wave, v);
#pragma unroll
        for (int i = 0; i < kFirst / 64; ++i)
            s_key[wave * kFirst + 64 * i + lane] = v[i].x, s_index[wave * kFirst + 64 * i + lane] = (int)v[i].y;
    }
    start(s);
    const uint32_t top = top_of<T>(sp, b, s.key);
    if (top == 0) {
        if (t == 0) put(a, b, -1, 0, 0);
        return;
    }
    const Row row(set.t, top, s.powers);
    if (row.greedy) {   // in the first stretch that has it
        uint32_t from_end = 0;
        for (int i = t; i < sp.scans; i += T)
            if (sp.top[(int64_t)b * sp.scans + i] == top) from_end = max(from_end, (uint32_t)(sp.scans - i));
        const int first = (sp.scans - largest<T>(from_end, s.key)) * sp.scan;
        from_end = 0;
        for (int i = t; i < sp.scan; i += T)
            if (src.one(first + i) == top) from_end = max(from_end, (uint32_t)(sp.scan - i));
        from_end = largest<T>(from_end, s.key);
        if (t == 0) put(a, b, first + sp.scan - from_end, 1, 1);
        return;
    }
    uint64_t live = 0, all = 0;
    static_assert(T == 2 * kBins, "");
    if (t < kBins) {
#pragma unroll 8
        for (int c = 0; c < sp.chunks; ++c) live += counts[c * kBins + t];
        s.count[0][t] = (uint32_t)live;
    } else {
#pragma unroll 8
        for (int c = 0; c < sp.chunks; ++c) all += masses[c * kBins + t - kBins];
        s.mass[0][t - kBins] = all;
    }
    if (cut_at_all) {   // the first bins whose tokens all chunks list
        for (int c = t; c < sp.chunks; c += T) s_listed_of[c] = sp.listed[(int64_t)b * sp.chunks + c];
        if (t == 0) s_bins = kBins;
        __syncthreads();
        for (int c = t; c < sp.chunks; c += T) atomicMin(&s_bins, s_listed_of[c].x);
    }
    scan<T>(&live, &all, s.part);
    if (t == T - 1) s.found[0] = live, s.found[1] = all;
    __syncthreads();
    live = s.found[0], all = s.found[1];
    __syncthreads();

    // The tokens of a bin: among those that are listed; or gathered in LDS; or where they are too many read again
    // each time.
    enum { kListed, kGathered, kReadAgain } from = kReadAgain;
    int bin = -1;
    auto stream = [&](auto f) {   // eight reads under way
        constexpr int N = 8;
        for (int c = wave; c < sp.chunks; c += WAVES) {
            const int end = min(a.vocab, (c + 1) * kChunk);
#pragma unroll 1
            for (int i0 = c * kChunk + 4 * lane; i0 - 4 * lane < end; i0 += 256 * N) {
                uint32_t key[N][4];
#pragma unroll
                for (int n = 0; n < N; ++n) src.four(i0 + 256 * n, key[n]);
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) f(key[n][e], i0 + 256 * n + e, c);
            }
        }
    };
    auto prepare = [&](int next, uint64_t count) {
        if (next == bin) return;
        bin = next;
        from = bin < s_bins ? kListed : count <= kList ? kGathered : kReadAgain;
        if (from != kGathered) return;
        held = false;
        __syncthreads();
        if (t == 0) s_listed = 0;
        __syncthreads();
        stream([&](uint32_t k, int i, int) {
            if (k && row.bin(k) == bin) {
                const uint32_t at = atomicAdd(&s_listed, 1u);
                if (at < kList) s_key[at] = k, s_index[at] = i;
            }
        });
        __syncthreads();
    };
    auto each_token = [&](auto f) {
        if (from == kListed) {
            for (int c = wave; c < sp.chunks; c += WAVES) {
                const int n = s_listed_of[c].y;
                if (held) {
                    for (int i = lane; i < n; i += 64) f(s_key[c * kFirst + i], s_index[c * kFirst + i]);
                    continue;
                }
                uint2 v[kFirst / 64];
                read_list(c, v);
#pragma unroll
                for (int i = 0; i < kFirst / 64; ++i)
                    if (64 * i + lane < n) f(v[i].x, (int)v[i].y);
            }
        } else if (from == kGathered) {
            for (uint32_t i = t; i < min(s_listed, (uint32_t)kList); i += T) f(s_key[i], s_index[i]);
        } else {
            stream([&](uint32_t k, int i, int) { if (k) f(k, i); });
        }
    };
    const Kept kept = cut(set, s, row, live, prepare, each_token,
                          [&](const Kept &, bool by_k, const Found &in) { return by_k ? in.mass_before : all; });

    // What is kept of each chunk: whole bins, and of the one where the cut is the tokens that are kept.
    const bool cuts = kept.key > kLeast || kept.index != 0xffffffffu;
    const int last = cuts ? row.bin(kept.key) : kBins;
    for (int c = t; c < MOST; c += T) s_chunk[c] = 0;
    __syncthreads();
    for (int c = wave; c < sp.chunks; c += WAVES) {
        uint64_t m = 0;
        for (int i0 = 0; i0 < last; i0 += 256)
#pragma unroll
            for (int i = i0 + lane; i < i0 + 256; i += 64) {
                const uint64_t v = masses[c * kBins + i];
                m += i < last ? v : 0;
            }
        m = wave_all(m, Sum());
        if (lane == 0) s_chunk[c] = m;
    }
    __syncthreads();
    if (cuts) {
        prepare(last, s.count[0][last]);   // another bin where the last cut was that of min_p
        if (from != kReadAgain) {
            each_token([&](uint32_t k, int i) {
                if (kept.has(k, i) && row.bin(k) == last) atomicAdd((unsigned long long *)&s_chunk[i / kChunk], (unsigned long long)row.mass(k));
            });
        } else {
            for (int c = wave; c < sp.chunks; c += WAVES) {
                uint64_t m = 0;
                for (int i = c * kChunk + 4 * lane; i < min(a.vocab, (c + 1) * kChunk); i += 256) {
                    uint32_t key[4];
                    src.four(i, key);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (kept.has(key[e], i + e) && row.bin(key[e]) == last) m += row.mass(key[e]);
                }
                m = wave_all(m, Sum());
                if (lane == 0) s_chunk[c] += m;   // the wave's own
            }
        }
        __syncthreads();
    }
    uint64_t total = 0;
    for (int c = 0; c < sp.chunks; ++c) total += s_chunk[c];
    const uint64_t target = place_of(set.u, total);
    uint64_t before = 0;
    int c = 0;
    for (; c < sp.chunks - 1 && before + s_chunk[c] <= target; ++c) before += s_chunk[c];
    // the chunk again, eight tokens a thread
    uint32_t key[8];
    uint64_t m[8], mine = 0;
    const int i0 = c * kChunk + 8 * t;
    src.four(i0, key), src.four(i0 + 4, key + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) mine += m[e] = key[e] && kept.has(key[e], i0 + e) ? row.mass(key[e]) : 0;
    uint64_t upto = mine, none = 0;
    scan<T>(&upto, &none, s.part);
    upto += before - mine;
    if (upto > target || upto + mine <= target) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (upto <= target && upto + m[e] > target) put(a, b, i0 + e, m[e], total);
        upto += m[e];
    }
}

template <typename E, bool ALONG> hipError_t run_row(const SampleArgs &a, hipStream_t st) {
    // As many threads as keep each busy: 1000 tokens take 8.4 us with 256 threads and 8.7 with 512 (and with 128 a fifth
    // more than with 256), 4000 tokens 20.8 with 256, 16.6 with 512 and 17.8 with 1024, 8000 tokens 20.9 and 20.6.
    if (a.vocab <= 1024) k_sample_row<E, ALONG, 256, 1024><<<a.batch, 256, 0, st>>>(a);
    else if (a.vocab <= 8192) k_sample_row<E, ALONG, 512, 8192><<<a.batch, 512, 0, st>>>(a);
    else k_sample_row<E, ALONG, 1024, kRow><<<a.batch, 1024, 0, st>>>(a);
    return hipGetLastError();
}
template <typename E> hipError_t run_long(const SampleArgs &a, const Space &sp, hipStream_t st) {
    k_sample_bins<E><<<dim3(sp.chunks, a.batch), 512, 0, st>>>(a, sp);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    k_sample_pick<E><<<a.batch, 1024, 0, st>>>(a, sp);
    return hipGetLastError();
}

// Rows whose elements lie apart are read as they lie up to so many tokens, each element a line of its own: 16 rows of 4000
// tokens 19.6 us and laid out first 23.3, 64 rows 20.5 and 24.2; 64 rows of 8000 29.3 laid out and 31.5, of 30000 45
// and 66.
constexpr int kApart = 4096;

template <typename E> hipError_t run(SampleArgs a, hipStream_t st) {
    const bool along = a.token_stride == 1;
    const Space sp = space_of(a.workspace, a.batch, a.vocab, !along);
    if (a.vocab <= kRow && (along || a.vocab <= kApart)) return along ? run_row<E, true>(a, st) : run_row<E, false>(a, st);
    if (along) {
        k_sample_scan<E><<<dim3(sp.scans, a.batch), 256, 0, st>>>(a, sp);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        return run_long<E>(a, sp, st);
    }
    k_sample_lay<E><<<dim3(sp.scans, (a.batch + 15) / 16), 256, 0, st>>>(a, sp);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.logits = sp.keys, a.row_stride = sp.row, a.token_stride = 1;
    return a.vocab <= kRow ? run_row<uint32_t, true>(a, st) : run_long<uint32_t>(a, sp, st);
}

}  // namespace

// Whatever the strides are.
int64_t sample_workspace(int batch, int vocab) { return vocab <= kApart ? 0 : space_of(nullptr, batch, vocab, true).bytes; }

hipError_t launch_sample(const SampleArgs &a, hipStream_t st) {
    return a.dtype == BSP_F32 ? run<float>(a, st) : run<uint16_t>(a, st);
}

}  // namespace bsp
