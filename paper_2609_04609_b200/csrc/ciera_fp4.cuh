// Codes and scale bytes of 4-bit operands.
#pragma once

#include "ciera_numeric.cuh"

namespace ciera {

constexpr uint32_t kAtomBytes = 512;  // scale bytes of 128 rows and 128 columns

// The scale byte of a group whose largest magnitude has these bits: the least s >= -126 with amax <= 1.5 * 2^2 * 2^s.
__device__ __forceinline__ uint32_t scale_byte4(uint32_t amax) {
    if (amax >= 0x7f800000u) return 255u;
    if (amax == 0u) return 127u;
    return (uint32_t)max((int)((amax + 0x3fffffu) >> 23) - 2, 1);  // (a mantissa above 1.5 carries into the exponent)
}
// 2^s for a scale byte s + 127; NaN for byte 255
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}
// where in its atom the four bytes of a row begin
__host__ __device__ constexpr uint32_t atom_word(uint32_t row) { return (row & 31u) * 16u + (row >> 5 & 3u) * 4u; }
// eight codes as four pairs of fp16 values, the first in the low halves
__device__ __forceinline__ void from_e2m1x8(uint32_t codes, uint32_t (&two)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(two[0]), "=r"(two[1]), "=r"(two[2]), "=r"(two[3])
        : "r"(codes));
}

}  // namespace ciera
