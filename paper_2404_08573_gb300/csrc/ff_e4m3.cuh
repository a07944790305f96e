// Blocks of e4m3 values with an fp32 scale: what writes them agrees on these.
#pragma once

#include <cuda_fp8.h>

#include "ff_internal.cuh"

namespace ff {

constexpr float kE4m3Max = 448.f;
constexpr float kScaleMin = 1.17549435e-38f;  // 2^-126

// The scale of a block whose largest magnitude has these bits (the bits of
// non-negative floats order like the floats, with infinity and then NaN above
// all of them, so an integer maximum keeps both).
__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
  const float s = __fdiv_rn(__uint_as_float(amax_bits), kE4m3Max);
  return s < kScaleMin ? kScaleMin : s;  // keeps NaN
}

// Two values as e4m3 (to nearest even, saturating; NaN stays NaN), a in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

}  // namespace ff
