// The next token of rows of logits: temperature, top-k, top-p and min-p, by given random numbers.
//
// What is kept is always the first of the tokens in order (falling logit, rising index), so that it is
// told by a logit and by how many of the tokens that have just it are kept.  Both are found without a sort, by
// counting and by adding up whole numbers, which has no order that could show.
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"

namespace bsp {

namespace {

constexpr int kRowThreads = 1024, kWaves = kRowThreads / 64;
constexpr double kOne = 8796093022208.0;   // 2^43: what a weight of 1 counts; 2^20 of them stay below 2^63

// Logits as numbers that are in the same order; NaN and -Inf, which are never taken, are 0.
__device__ __forceinline__ uint32_t key_of(float l) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t u = __float_as_uint(l + 0.f);   // -0 as 0
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return key == 0 ? -INFINITY : __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}

struct Row {
    float top;        // the largest logit
    double inv;       // 1 / temperature; 0 for the largest logit only
    bool greedy;
    __device__ __forceinline__ double weight(float l) const {   // in units of 1
        if (l == top) return 1.0;
        if (greedy || !(l > -INFINITY) || top == INFINITY) return 0.0;
        return exp(((double)l - top) * inv);
    }
    __device__ __forceinline__ uint64_t mass(float l) const { return (uint64_t)rint(weight(l) * kOne); }
};

// Sum over the workgroup, for all its threads.
template <typename T> __device__ __forceinline__ T sum_of(T v, T *s_part) {
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if (threadIdx.x % 64 == 0) s_part[threadIdx.x / 64] = v;
    __syncthreads();
    T all = 0;
    for (int w = 0; w < kWaves; ++w) all += s_part[w];
    return all;
}

// A row's tokens down to a logit, and of those that have it the first `equal`.
struct Kept {
    uint32_t key;
    uint32_t equal;
};

// A workgroup for a row, which is read again for each step.
template <typename E> __global__ __launch_bounds__(kRowThreads) void k_sample(SampleArgs a) {
    __shared__ uint64_t s_part[kWaves], s_mass[256], s_seg[kWaves + 1];
    __shared__ uint32_t s_count[256], s_pick[2];
    __shared__ uint64_t s_rest;
    const int b = blockIdx.x, t = threadIdx.x, lane = t % 64, wave = t / 64;
    const E *row = (const E *)a.logits + b * a.row_stride;
    auto logit = [&](int i) { return logit_of(key_of(to_f32(row[i * a.token_stride]))); };

    Row r;
    uint32_t top = 0;
    for (int i = t; i < a.vocab; i += kRowThreads) top = max(top, key_of(to_f32(row[i * a.token_stride])));
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if (lane == 0) s_count[wave] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = max(top, s_count[w]);
    if (top == 0) {
        if (t == 0) {
            a.tokens[b] = -1;
            if (a.logp) a.logp[b] = -INFINITY;
        }
        return;
    }
    r.top = logit_of(top);
    const float temperature = a.temperature ? a.temperature[b] : 1.f;
    r.greedy = !(temperature > 0.f);
    r.inv = 1.0 / temperature;

    // The tokens up to which `target` tokens, or that much mass, come together, among the kept ones; by
    // 8 bits of the key at a time.
    Kept kept = {1, 0xffffffffu};
    auto select = [&](bool by_mass, uint64_t target) {
        uint32_t prefix = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (t < 256) s_count[t] = 0, s_mass[t] = 0;
            __syncthreads();
            for (int i = t; i < a.vocab; i += kRowThreads) {
                const float l = logit(i);
                const uint32_t key = key_of(l);
                if (key < kept.key || (shift < 24 && key >> (shift + 8) != prefix >> (shift + 8))) continue;
                atomicAdd(&s_count[key >> shift & 255], 1u);
                if (by_mass) atomicAdd((unsigned long long *)&s_mass[key >> shift & 255], (unsigned long long)r.mass(l));
            }
            __syncthreads();
            if (t == 0) {
                uint64_t before = 0;
                int bin = 255;
                // of the last kept logit only some tokens are kept: the last bin may hold less than it says,
                // which matters to no one as the target does not exceed what is kept
                for (; bin > 0; --bin) {
                    const uint64_t here = by_mass ? s_mass[bin] : s_count[bin];
                    if (before + here >= target) break;
                    before += here;
                }
                s_pick[0] = bin, s_pick[1] = s_count[bin], s_rest = before;
            }
            __syncthreads();
            prefix |= s_pick[0] << shift;
            target -= s_rest;
        }
        Kept k;
        k.key = prefix;
        if (by_mass) {
            const uint64_t one = r.mass(logit_of(prefix));
            target = one ? (target + one - 1) / one : s_pick[1];
        }
        k.equal = (uint32_t)min((uint64_t)s_pick[1], max((uint64_t)1, target));
        if (k.key == kept.key) k.equal = min(k.equal, kept.equal);
        kept = k;
    };
    const int top_k = a.top_k ? a.top_k[b] : 0;
    if (r.greedy) {
        kept = {top, 1};
    } else if (top_k > 0 && top_k < a.vocab) {
        uint64_t live = 0;
        for (int i = t; i < a.vocab; i += kRowThreads) live += key_of(to_f32(row[i * a.token_stride])) != 0;
        if (sum_of(live, s_part) > (uint64_t)top_k) select(false, top_k);
    }
    const float top_p = a.top_p ? a.top_p[b] : 1.f;
    if (!r.greedy && top_p < 1.f) {
        uint64_t mass = 0, equal = 0;
        for (int i = t; i < a.vocab; i += kRowThreads) {
            const float l = logit(i);
            const uint32_t key = key_of(l);
            if (key > kept.key) mass += r.mass(l);
            equal += key == kept.key;
        }
        mass = sum_of(mass, s_part), equal = sum_of(equal, s_part);
        mass += min(equal, (uint64_t)kept.equal) * r.mass(logit_of(kept.key));
        select(true, max((uint64_t)1, (uint64_t)ceil(fmax((double)top_p, 0.0) * (double)mass)));
    }
    const float min_p = a.min_p ? a.min_p[b] : 0.f;
    auto likely = [&](float l) { return l == r.top || !(r.weight(l) < min_p); };   // NaN: no cut

    // Each wave adds up what is kept of a stretch of the row; then the wave of the stretch in which the sum
    // passes u looks for the token.
    const int per = (a.vocab + kWaves * 64 - 1) / (kWaves * 64) * 64;
    const int from = min(a.vocab, wave * per), to = min(a.vocab, from + per);
    uint32_t equal = 0;
    uint64_t above = 0;
    const uint64_t one = likely(logit_of(kept.key)) ? r.mass(logit_of(kept.key)) : 0;
    for (int i = from + lane; i < to; i += 64) {
        const float l = logit(i);
        const uint32_t key = key_of(l);
        equal += key == kept.key;
        if (key > kept.key && likely(l)) above += r.mass(l);
    }
    for (int d = 1; d < 64; d *= 2) equal += __shfl_xor(equal, d), above += __shfl_xor(above, d);
    __syncthreads();
    if (lane == 0) s_count[wave] = equal, s_seg[wave] = above;
    __syncthreads();
    uint32_t seen = 0;   // of the last logit, before this wave
    uint64_t before = 0, total = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = total;
        const uint32_t upto = min(kept.equal, seen + s_count[w]);
        total += s_seg[w] + (upto - min(kept.equal, seen)) * one;
        seen += s_count[w];
    }
    seen = 0;
    for (int w = 0; w < wave; ++w) seen += s_count[w];
    const float u = fminf(fmaxf(a.u[b], 0.f), 0x1.fffffep-1f);
    const uint64_t target = (uint64_t)((double)u * (double)total);   // the sum has to be more
    uint64_t mine = s_seg[wave] + (min(kept.equal, seen + s_count[wave]) - min(kept.equal, seen)) * one;
    if (target < before || target >= before + mine) return;
    for (int i0 = from; i0 < to; i0 += 64) {
        const int i = i0 + lane;
        const float l = i < to ? logit(i) : -INFINITY;
        const uint32_t key = key_of(l);
        const uint64_t same = __ballot(key == kept.key);
        const uint32_t rank = seen + __popcll(same & ((1ull << lane) - 1));
        const uint64_t m = key == kept.key ? (rank < kept.equal ? one : 0) : key > kept.key && likely(l) ? r.mass(l) : 0;
        uint64_t upto = m;
        for (int d = 1; d < 64; d *= 2) {
            const uint64_t o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const uint64_t hit = __ballot(before + upto > target);
        if (hit) {
            if (lane == __ffsll((unsigned long long)hit) - 1) {
                a.tokens[b] = i;
                if (a.logp) a.logp[b] = (float)log((double)m / (double)total);
            }
            return;
        }
        before += __shfl(upto, 63);
        seen += __popcll(same);
    }
}

}  // namespace

int64_t sample_workspace(int, int) { return 0; }

hipError_t launch_sample(const SampleArgs &a, hipStream_t st) {
    if (a.dtype == BSP_F32)
        k_sample<float><<<a.batch, kRowThreads, 0, st>>>(a);
    else
        k_sample<uint16_t><<<a.batch, kRowThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace bsp
