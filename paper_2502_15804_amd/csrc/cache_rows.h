// Where the tokens of a pair lie in a growing cache: one run of rows (packed), or pages of rows (paged).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "fairkv.h"

namespace fairkv {

constexpr int kCacheScales = FAIRKV_CACHE_SCALES;

// What a kernel needs to find a token's row.  One of off and pages is null.
struct RowMap {
    const int64_t *off;      // [pairs]
    const int32_t *pages;    // [pairs][max_pages]
    int64_t n_rows;
    int32_t max_pages, page_shift;

    // Row of token t >= 0 of a pair, or -1 where it has none in the cache.
    __device__ __forceinline__ int64_t row(int64_t pair, int32_t t) const
    {
        if (!pages) {
            const int64_t first = off[pair];
            return first >= 0 && static_cast<uint64_t>(first) + static_cast<uint32_t>(t) < static_cast<uint64_t>(n_rows) ? first + t : -1;
        }
        const int32_t page = t >> page_shift;
        if (page >= max_pages) return -1;
        return row_of_page(pages[pair * max_pages + page], t);
    }
    // The same, of a token of the page `id`.
    __device__ __forceinline__ int64_t row_of_page(int32_t id, int32_t t) const
    {
        const int64_t first = static_cast<int64_t>(id) << page_shift;
        return id >= 0 && first + (1 << page_shift) <= n_rows ? first + (t & ((1 << page_shift) - 1)) : -1;
    }
};

}  // namespace fairkv
