// 8-bit floating point (e4m3: four exponent bits, bias 7, three mantissa bits, largest 448, no infinity) on the device.
#pragma once
#include "sqnn_decode.cuh"

#include <cuda_bf16.h>

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

SQNN_DEV uint32_t bf16x2(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return reinterpret_cast<const uint32_t &>(b);
}

}  // namespace sqnn
