// What the kernels of the paged int8 cache share: the cache and the batch as they see them, a sequence's new tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_plans.hpp"
#include "kernels.hpp"
#include "number_formats.hpp"

namespace dessert {

constexpr uint32_t NO_PAGE = 0xFFFFFFFFu;

// A barrier with the wave's LDS operations waited for.  (The compiler leaves the wait out of barriers at the heads of some loops, over whose back
// edges LDS operations come.)
__device__ inline void barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// A sequence's new tokens: rows first .. first + count, at positions begin .. begin + count (negative ones are nowhere).
struct NewTokens {
    uint32_t first, count;
    int32_t begin;
};

__device__ inline NewTokens new_tokens(const CacheBatch& b, uint32_t s) {
    NewTokens n;
    if (b.starts) {
        const uint32_t lo = b.starts[s], hi = b.starts[s + 1];
        const uint32_t all = min(hi > lo ? hi - lo : 0u, CACHE_MOST);
        n.first = min(lo, b.n_tokens);
        n.count = min(all, min(b.n_tokens - n.first, b.max_tokens));
        n.begin = (int32_t)min(b.lengths[s], CACHE_MOST) - (int32_t)all;
    } else {
        n.first = s;
        n.count = 1;
        n.begin = (int32_t)min(b.lengths[s], CACHE_MOST) - 1;
    }
    return n;
}

// The page at a place of a sequence's table, or NO_PAGE: behind the table's end, or no number of this pool.
__device__ inline uint32_t page_at(const CacheBatch& b, const uint32_t* table, uint32_t place, uint32_t n_pages) {
    const uint32_t page = table[min(place, b.table_pages - 1)];     // loaded in any case: no branch for the loads behind it to wait at
    return place < b.table_pages && page < n_pages ? page : NO_PAGE;
}

}  // namespace dessert
