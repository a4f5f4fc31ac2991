// Helpers of the sources behind vmoe_train.h (gfx950 only).
#pragma once

#include "../../include/vmoe_train.h"
#include "common.h"

namespace vmoe {

template <int CTRL, int ROWS>
__device__ __forceinline__ float add_dpp(float v) {
    const int moved = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF,
                                                  false);
    return v + __builtin_bit_cast(float, moved);
}

// Sum over a wave's 64 lanes, the same value (a scalar) for all: sums run up
// each row of 16 lanes, then over the rows, into lane 63. All lanes active.
__device__ __forceinline__ float wave_total(float v) {
    v = add_dpp<0x111, 0xF>(v);  // row_shr:1, 2, 4, 8
    v = add_dpp<0x112, 0xF>(v);
    v = add_dpp<0x114, 0xF>(v);
    v = add_dpp<0x118, 0xF>(v);
    v = add_dpp<0x142, 0xA>(v);  // lane 15 of rows 0, 2 to rows 1, 3
    v = add_dpp<0x143, 0xC>(v);  // lane 31 to rows 2, 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

}  // namespace vmoe
