// Which tile, or half of one, a workgroup takes where tiles fill a compute unit each: those of a last round that is at most half full are
// halved between two workgroups.  Code of host and device, without HIP.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define IWP_BOTH __host__ __device__
#else
#define IWP_BOTH
#endif

namespace iwp {

constexpr uint32_t TILES_AT_A_TIME = 256;              // compute units
constexpr uint32_t MOST_HALVES = TILES_AT_A_TIME / 2;  // workgroups that halves add to a launch

struct TilePart {
    uint32_t tile;
    uint32_t half;         // 0: the whole tile, 1: the upper half, 2: the lower
};
// false: there is nothing for this workgroup.  whole: tiles that are not halved.
IWP_BOTH inline bool part_of(uint32_t block, uint32_t tiles, TilePart* part, uint32_t* whole) {
    const uint32_t last = tiles % TILES_AT_A_TIME, halved = last <= TILES_AT_A_TIME / 2 ? last : 0;
    *whole = tiles - halved;
    if (block < *whole) {
        *part = TilePart{block, 0};
        return true;
    }
    const uint32_t half = block - *whole;
    *part = TilePart{*whole + half / 2, 1 + half % 2};
    return half < 2 * halved;
}

}  // namespace iwp

#undef IWP_BOTH
