// Sums over a wavefront's 64 lanes by data-parallel primitives: six vector instructions, where shuffles go through LDS six times
// (a find_tile of packed.h takes one sum after the other, one and another each time the longest sequence's tiles double: 6 for 4096 rows
// in 128-row tiles, 11 for 32768 in 32-row ones).
#pragma once
#include <hip/hip_runtime.h>

namespace sa {

// x of the lane that CTRL names, 0 where there is none or ROWS (of 16 lanes, a bit each) leaves the row out
template <int CTRL, int ROWS = 15>
__device__ inline int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 15, false); }
// sum over this lane and those before it
__device__ inline int wave_scan(int x) {
    x += from_lane<0x111>(x);           // one, two, four and eight lanes to the left, within a row
    x += from_lane<0x112>(x);
    x += from_lane<0x114>(x);
    x += from_lane<0x118>(x);
    x += from_lane<0x142, 10>(x);       // last lane of the row before, to rows 1 and 3
    x += from_lane<0x143, 12>(x);       // lane 31, to rows 2 and 3
    return x;
}
// sum over all lanes, in a scalar register
__device__ inline int wave_total(int scanned) { return __builtin_amdgcn_readlane(scanned, 63); }

}  // namespace sa
