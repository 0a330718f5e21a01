// Rounding to e4m3 codes with a power of two as their scale.
#pragma once

#include "common.cuh"

namespace gbmoe {

// Exponent of the smallest power of two 2^e (e >= -127) with amax <= 448 * 2^e
__device__ __forceinline__ int scale_exponent(float amax) {
    int x;
    const float m = frexpf(amax, &x);  // amax = m * 2^x, m in [0.5, 1); 448 = 0.875 * 2^9
    if (amax == 0.0f) return -127;
    return max(x - 9 + (m > 0.875f ? 1 : 0), -127);
}

// 2^e for e in -127 .. 127 (subnormal at -127)
__device__ __forceinline__ float pow2(int e) { return e > -127 ? __uint_as_float((uint32_t)(e + 127) << 23) : __uint_as_float(0x00400000u); }

// two fp32 -> two e4m3 bytes (low byte: a), nearest, ties to even, +-448 beyond
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ uint2 e4m3x8(const float (&v)[8], float s) {
    return make_uint2(e4m3x2(v[0] * s, v[1] * s) | e4m3x2(v[2] * s, v[3] * s) << 16,
                      e4m3x2(v[4] * s, v[5] * s) | e4m3x2(v[6] * s, v[7] * s) << 16);
}

}  // namespace gbmoe
