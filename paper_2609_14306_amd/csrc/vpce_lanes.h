// Values of other lanes of a wavefront without a trip through LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vpce {

// v of another lane through the data-parallel path (CTRL: the lane selection), 0 where
// the selection has no lane or ROWS leaves the lane's row of 16 out.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int lane_move(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double lane_move(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)lane_move<CTRL, ROWS>((int)(uint32_t)u);
  const uint32_t hi = (uint32_t)lane_move<CTRL, ROWS>((int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
  return __int_as_float(lane_move<CTRL>(__float_as_int(v)));
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e;                            // lane ^ 1, lane ^ 2
constexpr int kHalfMirror = 0x141, kMirror = 0x140;                    // 7 - lane in 8, 15 - lane in 16
constexpr int kUp1 = 0x111, kUp2 = 0x112, kUp4 = 0x114, kUp8 = 0x118;  // lane - n in 16
constexpr int kRowEnd = 0x142, kHalfEnd = 0x143;  // last lane of the row / the half in front

__device__ __forceinline__ float lane_read(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ double lane_read(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

}  // namespace vpce
