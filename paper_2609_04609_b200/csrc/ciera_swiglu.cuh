// silu(g) * u in 32 bits.
#pragma once

#include "ciera_numeric.cuh"

namespace ciera {

// sigmoid(g) = 1 / (1 + e) and 1 - sigmoid(g) = e / (1 + e) with e = 2^(-g log2 e): the exponent in two parts (log2 e as the nearest
// 32-bit number and what is left of it), so that the power is off by a step or two however large the exponent is, and both
// results by less than 2^-21 of themselves; for g above 87 e and 1 - sigmoid(g) are 0.  Gates below kLowestGate, where e leaves 32
// bits, are not for this.  (expf and a division: silu(g) * u of 32768 x 1024 in 93 us.)
constexpr float kLowestGate = -87.f;
__device__ __forceinline__ float2 sigmoid32(float g) {
    const float x = fminf(fmaxf(g, kLowestGate), 127.f), t = x * -1.44269504f;
    const float rest = fmaf(x, -1.44269504f, -t) + x * -1.92596299e-8f;  // -x log2 e = t + rest
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    e = fmaf(e, rest * 0.693147181f, e);
    float s;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    return make_float2(s, e * s);  // (a NaN is not seen here; g itself is a factor of all that this goes into)
}
__device__ __forceinline__ float swiglu32(float g, float u) { return g * sigmoid32(g).x * u; }
// The same with the gate last: g * sigmoid(g) of a gate below 2^-126 has lost bits, of the least one all, which a large u would bring back,
// while sigmoid(g) * u is below 2^-126 only where the result counts for nothing beside the least power of two of a group.
__device__ __forceinline__ float swiglu32_any(float g, float u) { return g * (sigmoid32(g).x * u); }

}  // namespace ciera
