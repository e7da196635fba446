// 8-bit floating point (e4m3: four exponent bits, bias 7, three mantissa bits, largest 448, no infinity) on the device.
#pragma once
#include "sqnn_decode.cuh"

namespace sqnn {

constexpr uint32_t FP8_BLOCK = SQNN_FP8_BLOCK;   // columns (and, of weights, rows) that share a scale
constexpr float FP8_MAX = 448.0f;

// Two fp32 numbers to e4m3, to nearest even, larger ones to the largest; `lo` in the low byte.
SQNN_DEV uint32_t to_fp8x2(float lo, float hi)
{
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(v) : "f"(hi), "f"(lo));
    return v;
}

// Whether an fp32 number within 448 lies within six of its last places of the middle between two neighbouring e4m3 numbers.  Above
// 2^-6 a middle is where the 20 bits behind the three kept are 1000...; below, where e4m3 numbers are 2^-9 apart, 2^-6 is
// added first: that puts the number where the spacing is the same.
SQNN_DEV bool near_fp8_border(float t)
{
    float a = fabsf(t);
    a = a < 0x1p-6f ? a + 0x1p-6f : a;
    const uint32_t behind = __float_as_uint(a) & 0xfffffu;
    return behind - (0x80000u - 6u) <= 12u;
}

}  // namespace sqnn
