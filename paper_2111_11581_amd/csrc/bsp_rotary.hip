// Rotary positions, with norms of heads in the same pass and the write of keys and values into a
// paged cache.
#include <hip/hip_runtime.h>

#include "bsp_decode.h"
#include "bsp_decode_dev.h"
#include "bsp_paged.h"

namespace bsp {

namespace {

struct Turn {
    float cos, sin;
};
// Cosine and sine of pos * freq.  Whole turns are taken off in fp64, where the angle of a position up to
// 2^31 keeps 2^-22 radians and one up to 2^20 2^-33; what fp32 cannot hold of the rest, in half turns, turns the
// result by itself.
__device__ __forceinline__ Turn turn(int pos, double freq) {
    double t = pos * freq * 0.15915494309189533577;   // 1 / 2 pi: turns
    t = 2.0 * (t - rint(t));
    const float half = (float)t, rest = (float)(t - half) * 3.14159265358979f;
    float s, c;
    sincospif(half, &s, &c);
    return {c - s * rest, s + c * rest};
}

// A wave for a head of a token: queries, keys, values.
template <typename E> __global__ __launch_bounds__(64) void k_rotary(RotaryArgs a) {
    const int i = blockIdx.x, lane = threadIdx.x, D = a.head_dim, half = a.rope.dims / 2;
    int h = blockIdx.y;
    const int pos = a.pos[i];
    const E *src;
    E *dst;
    int64_t from, to;   // strides of dimensions
    const float *norm = nullptr;
    bool rotated = true;
    if (h < a.heads) {
        src = (const E *)a.x + i * a.xs.seq + h * a.xs.head, from = a.xs.dim;
        dst = (E *)a.y + i * a.ys.seq + h * a.ys.head, to = a.ys.dim;
        norm = a.x_norm;
    } else {
        h -= a.heads;
        const bool value = h >= a.kv_heads;
        if (value) h -= a.kv_heads;
        const int64_t at = place_of(a.c, a.table, a.rows ? a.rows[i] : i, a.seqs, a.width, pos);
        if (at < 0) return;
        const bsp_strides s = value ? a.vs : a.ks;
        src = (const E *)(value ? a.v : a.k) + i * s.seq + h * s.head, from = s.dim;
        dst = (E *)(value ? a.values : a.keys) + at + h * a.c.head_stride, to = 1;
        norm = value ? nullptr : a.k_norm;
        rotated = !value;
    }
    // a lane's pairs, and its dimensions that are passed on: all are read before any is written
    const int pairs = rotated ? half : 0, rest = 2 * pairs;
    const bool beside = a.rope.layout == BSP_ROPE_INTERLEAVED;
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
        for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
        by = 1.f / sqrtf(sum / D + a.eps);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int p = lane + 64 * j, d0 = beside ? 2 * p : p, d1 = beside ? 2 * p + 1 : p + pairs;
        if (p >= pairs) break;
        if (norm) x[j][0] *= by * norm[d0], x[j][1] *= by * norm[d1];
        Turn t = turn(pos, a.freqs[p]);
        t.cos *= a.rope.factor, t.sin *= a.rope.factor;
        dst[d0 * to] = from_f32<E>(x[j][0] * t.cos - x[j][1] * t.sin);
        dst[d1 * to] = from_f32<E>(x[j][1] * t.cos + x[j][0] * t.sin);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int d = rest + lane + 64 * j;
        if (d < D) dst[d * to] = norm ? from_f32<E>(z[j] * (by * norm[d])) : whole[j];
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t st) {
    const dim3 grid(a.n, a.heads + 2 * a.kv_heads);
    if (a.dtype == BSP_F32)
        k_rotary<float><<<grid, 64, 0, st>>>(a);
    else
        k_rotary<uint16_t><<<grid, 64, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace bsp
