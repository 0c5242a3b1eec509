// Calls with more workgroups than a launch may have, as several launches (host code, no HIP).
#pragma once
#include <stdint.h>

#include <algorithm>

namespace dessert {

// A launch has fewer than 2^32 work-items in a dimension: a workgroup of 256 threads a row ends at 16 777 215 rows, which 288 GB can hold.
// launch(first, count, workgroups) for consecutive slices of n items, `per` items to a workgroup of `threads`; none for n = 0.
template <typename F>
void in_launches(uint64_t n, uint64_t per, uint32_t threads, F launch) {
    const uint64_t most = 0xFFFFFFFFull / threads * per;
    for (uint64_t first = 0; first < n; first += most) {
        const uint64_t count = std::min(most, n - first);
        launch(first, count, (uint32_t)((count + per - 1) / per));
    }
}

}  // namespace dessert
