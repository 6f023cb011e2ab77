// Launches over rows of a matrix, whose workgroups can be more than a launch takes.  Host code without HIP.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace iwp {

// HIP counts the threads of a launch in 32 bits: 524288 rows of 131072 entries, 16 a thread, are one too many.
constexpr uint64_t MOST_THREADS = 0xffffffffu;

// f(first row, workgroups) for launches of `threads` to a workgroup that take rows_per_block rows by `across` workgroups; the first result
// that is not 0, or 0.  across * threads fits 32 bits.  Only sizes beyond most memories take a second launch.
template <class F>
int in_launches(uint32_t rows, uint32_t rows_per_block, uint32_t across, uint32_t threads, F f) {
    const uint64_t most = MOST_THREADS / threads / across * rows_per_block;
    for (uint64_t row = 0; row < rows; row += most) {
        const uint32_t n = (uint32_t)std::min<uint64_t>(most, rows - row);
        if (int rc = f((uint32_t)row, (n + rows_per_block - 1) / rows_per_block * across)) return rc;
    }
    return 0;
}

}  // namespace iwp
