// Which tensor of a list a tile is in.
#pragma once

#include <stdint.h>

namespace mqg {

// The last of `count` (at least one, at most 1024) tensors that starts at or before `tile`; start[] ascends.  All lanes of a warp
// look at once, at every k-th tensor and then at k neighbours, with ordinary loads: a search by halves is ten dependent misses
// of the constant cache, which a launch begins without its parameters.  MANY: there may be more than 32.
template <bool MANY> __device__ __forceinline__ int find_in_list(const uint32_t* start, int count, uint32_t tile)
{
    asm volatile("" : "+l"(start));                     // an address like any other
    const int lane = threadIdx.x & 31, k = (count + 31) / 32;
    int base = 0;
    if (MANY && k > 1) {
        const uint32_t first = lane * k < count ? start[lane * k] : ~0u;
        base = (31 - __clz(__ballot_sync(0xFFFFFFFFu, first <= tile))) * k;
    }
    const uint32_t first = lane < k * (k == 1 ? 32 : 1) && base + lane < count ? start[base + lane] : ~0u;
    return base + 31 - __clz(__ballot_sync(0xFFFFFFFFu, first <= tile));
}

}  // namespace mqg
