// Where a token lies in a paged cache.
#pragma once
#include "bsp_decode.h"

namespace bsp {

// Page of token t of a sequence, or -1 where the entry holds nothing.
__device__ __forceinline__ int page_of(const CacheArgs &c, const int32_t *row, uint32_t t, uint32_t *slot) {
    const uint32_t e = fdiv(t, c.div_page);
    *slot = t - e * (uint32_t)c.page_size;
    const int p = row[e];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
}

// Element offset of position pos of a sequence's row within a plane, or -1 where it has no place.
__device__ __forceinline__ int64_t place_of(const CacheArgs &c, const int32_t *table, int row, int seqs, int width, int pos) {
    if ((unsigned)row >= (unsigned)seqs || pos < 0 || pos >= (int64_t)width * c.page_size) return -1;
    uint32_t slot;
    const int page = page_of(c, table + (int64_t)row * width, (uint32_t)pos, &slot);
    return page < 0 ? -1 : page * c.page_stride + slot * c.slot_stride;
}

}  // namespace bsp
