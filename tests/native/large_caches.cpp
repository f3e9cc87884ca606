// Which caches attention reads past the last-level cache, from the smallest to the largest that a call
// may name: more pages never turn it off again.
#include <cstdio>

#include "bsp_decode.h"

using namespace bsp;

int main() {
    int bad = 0;
    for (int dtype : {BSP_F32, BSP_BF16})
        for (int dim : {8, 128, 256})
            for (int64_t gap : {(int64_t)0, (int64_t)1 << 20})
                for (int64_t pages = 1; pages <= INT32_MAX; pages = pages * 2 + (pages % 3)) {
                    const int64_t stride = 16 * dim + gap;
                    const bsp_cache c = {dtype, BSP_HEAD_MAJOR, (int32_t)pages, 16, 1, dim, gap ? stride : 0};
                    const bool want = (unsigned __int128)2 * pages * stride * (dtype == BSP_F32 ? 4 : 2) > 128u << 20;
                    if (past_caches(cache_args(c)) != want) {
                        printf("dtype %d dim %d gap %lld pages %lld\n", dtype, dim, (long long)gap, (long long)pages);
                        ++bad;
                    }
                }
    // the largest page there can be, as often as can be
    const bsp_cache most = {BSP_F32, BSP_SLOT_MAJOR, INT32_MAX, INT32_MAX / 256, 1, 256, 0};
    if (!past_caches(cache_args(most))) ++bad, printf("most\n");
    return bad != 0;
}
