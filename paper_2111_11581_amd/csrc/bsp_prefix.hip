// Attention of one new token of each sequence over a paged cache, where groups of sequences share the
// pages of their first tokens.
#include <hip/hip_runtime.h>

#include <cmath>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"
#include "bsp_paged.h"

namespace bsp {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// A workgroup for a query head of a sequence, its waves in turn for the tokens.
template <typename E> __global__ __launch_bounds__(256) void k_prefix(PrefixArgs p) {
    const AttnArgs &a = p.a;
    __shared__ float s_m[4], s_l[4], s_o[4][256];
    const int h = blockIdx.x % a.heads, b = blockIdx.x / a.heads, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int D = a.c.head_dim, j = h / a.group;
    const int row = a.rows ? a.rows[b] : b;
    const bool in = (unsigned)row < (unsigned)a.seqs;
    const int len = in ? max(0, (int)min((int64_t)a.lens[row], (int64_t)a.width * a.c.page_size)) : 0;
    const int first = a.window && len > a.window ? len - a.window : 0;
    int shared = 0, prefix_row = -1;
    for (int g = 0; g < p.groups; ++g)
        if (b >= p.starts[g] && b < p.starts[g + 1]) {
            shared = p.shared[g];
            const int lead = p.starts[g];
            prefix_row = p.prefix_rows ? p.prefix_rows[g] : lead < 0 ? -1 : a.rows ? a.rows[lead] : lead;
            break;
        }
    const E *keys = (const E *)a.keys + j * a.c.head_stride, *values = (const E *)a.values + j * a.c.head_stride;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    for (int k = 0; k < 4; ++k) {
        const int d = lane + 64 * k;
        q[k] = d < D ? to_f32(((const E *)a.q)[b * a.qs.seq + h * a.qs.head + d * a.qs.dim]) : 0.f;
    }
    for (int t = first + wave; t < len; t += 4) {
        const int64_t at = place_of(a.c, a.table, t < shared ? prefix_row : row, a.seqs, a.width, t);
        if (at < 0) continue;
        float s = 0.f;
        for (int k = 0; k < 4; ++k) {
            const int d = lane + 64 * k;
            if (d < D) s += q[k] * to_f32(keys[at + d]);
        }
        for (int x = 1; x < 64; x *= 2) s += __shfl_xor(s, x);
        s *= a.scale * kLog2e;
        const float top = fmaxf(m, s), keep = exp2f(m - top), w = exp2f(s - top);
        m = top, l = l * keep + w;
        for (int k = 0; k < 4; ++k) {
            const int d = lane + 64 * k;
            if (d < D) o[k] = o[k] * keep + w * to_f32(values[at + d]);
        }
    }
    s_m[wave] = m, s_l[wave] = l;
    for (int k = 0; k < 4; ++k) s_o[wave][lane + 64 * k] = o[k];
    __syncthreads();
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, out = 0.f;
    for (int w = 0; w < 4; ++w) {
        const float f = exp2f(s_m[w] - ref);
        sum += s_l[w] * f, out += s_o[w][threadIdx.x] * f;
    }
    const int d = threadIdx.x;
    if (d < D) ((E *)a.y)[b * a.ys.seq + h * a.ys.head + d * a.ys.dim] = from_f32<E>(sum == 0.f ? 0.f : out / sum);
    if (d == 0 && a.lse) a.lse[(int64_t)b * a.heads + h] = (ref + log2f(sum)) * kLn2;
}

}  // namespace

int64_t prefix_workspace(const CacheArgs &, int, int, int, int) { return 0; }

hipError_t launch_prefix(const PrefixArgs &p, hipStream_t st) {
    if (p.a.c.dtype == BSP_F32)
        k_prefix<float><<<p.a.batch * p.a.heads, 256, 0, st>>>(p);
    else
        k_prefix<uint16_t><<<p.a.batch * p.a.heads, 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace bsp
