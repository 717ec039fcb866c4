// 8-bit floating point (e4m3: 4 exponent and 3 mantissa bits, largest value 448) with a power of two
// as scale for each block.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vpce_lanes.h"

namespace vpce {

// |v| if it is finite, else 0: what a block's scale goes by.
__device__ __forceinline__ float finite_magnitude(float v) {
  const float m = __builtin_fabsf(v);
  return m < INFINITY ? m : 0.f;
}

// Byte b of the scale 2^(b - 127): the smallest power of two with m <= 448 2^(b - 127).  448 is
// 1.75 2^8, so it is m's exponent less 8, or 7 where m's mantissa is above 1.75.
__device__ __forceinline__ int f8_scale(float m) {
  const uint32_t u = __float_as_uint(m);
  const int b = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
  return m == 0.f ? 127 : max(b, 0);
}
// 1 / 2^(b - 127), a normal number for every b that f8_scale gives.
__device__ __forceinline__ float f8_inverse(int b) { return __uint_as_float((uint32_t)(254 - b) << 23); }

// Four values, already over their scale, to the nearest, ties to even (the conversion's own rounding;
// the products with a power of two in front of it are exact); NaN for NaN and infinities.
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  auto fix = [](float v) { return __builtin_fabsf(v) < INFINITY ? v : __builtin_nanf(""); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(fix(a), fix(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(fix(c), fix(d), w, true);
  return (uint32_t)w;
}

// Maximum over 8, 16 or 32 consecutive lanes (from a multiple of as many), in each of them.
template <int LANES>
__device__ __forceinline__ float lanes_max(float m) {
  m = fmaxf(m, lane_move<kSwap1>(m));
  m = fmaxf(m, lane_move<kSwap2>(m));
  m = fmaxf(m, lane_move<kHalfMirror>(m));
  if constexpr (LANES >= 16) m = fmaxf(m, lane_move<kMirror>(m));
  if constexpr (LANES >= 32) m = fmaxf(m, __shfl_xor(m, 16));
  return m;
}

}  // namespace vpce
