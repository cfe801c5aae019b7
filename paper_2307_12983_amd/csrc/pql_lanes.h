// Sums over lanes of a wavefront whose number is known at run time.
#pragma once

#include <hip/hip_runtime.h>

namespace pql {

// Sum over groups of `lanes` consecutive lanes (a power of two; 64 and more: the wavefront), in one order for all of them: below
// 16 the partner's value comes with the addition itself (mirrors instead of the bits 4 and 8: lanes of one half hold equal
// sums by then).
__device__ __forceinline__ float lane_sum(float x, int lanes) {
#define PQL_LANE_ADD(CTRL) x += __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, 0xf, 0xf, false))
    if (lanes >= 2) PQL_LANE_ADD(0xB1);
    if (lanes >= 4) PQL_LANE_ADD(0x4E);
    if (lanes >= 8) PQL_LANE_ADD(0x141);
    if (lanes >= 16) PQL_LANE_ADD(0x140);
#undef PQL_LANE_ADD
    if (lanes >= 32) x += __shfl_xor(x, 16);
    if (lanes >= 64) x += __shfl_xor(x, 32);
    return x;
}

}  // namespace pql
