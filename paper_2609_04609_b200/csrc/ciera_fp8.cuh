// Scale bytes of 8-bit operands.
#pragma once

#include "ciera_numeric.cuh"

namespace ciera {

// The scale byte of a block whose largest magnitude has these bits: the least s >= -126 with amax <= 1.75 * 2^8 * 2^s.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax >= 0x7f800000u) return 255u;
    if (amax == 0u) return 127u;
    const int s = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(max(s, -126) + 127);
}

}  // namespace ciera
