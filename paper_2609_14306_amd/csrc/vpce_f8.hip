// Quantisation to 8 bits with block scales, for gfx950 (MI355X).  Bound by memory: every element is
// read once, held in registers while its block's largest magnitude is found, and written once.
// Eight lanes hold 128 columns of a row, 16 each, so that a lane writes 16 bytes.  16384 x 7168 of
// float32 in blocks of 1 x 128: 104 us, 5.7 TB/s; 25136 x 2880 of bfloat16 in blocks of 128 x 128: 41 us, 5.3
// TB/s (a 1 GiB copy: 5.2).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "vpce_f8.h"
#include "vpce_internal.h"

namespace vpce {

namespace {

constexpr int kRows = 32;  // rows that a workgroup of 256 takes side by side

// 16 elements from `p` on, as float32.
template <int DTYPE>
struct Sixteen {
  uint4 u[DTYPE == VP_BF16 ? 2 : 4];
  __device__ __forceinline__ void load(const void* X, int64_t element) {
    const uint4* p = (const uint4*)((const char*)X + element * (DTYPE == VP_BF16 ? 2 : 4));
#pragma unroll
    for (int k = 0; k < (int)(sizeof(u) / 16); ++k) u[k] = p[k];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(u) / 16); ++k) u[k] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ float get(int i) const {
    const uint4& v = u[DTYPE == VP_BF16 ? i / 8 : i / 4];
    if (DTYPE == VP_BF16) {
      const uint32_t w = i % 8 < 2 ? v.x : i % 8 < 4 ? v.y : i % 8 < 6 ? v.z : v.w;
      return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
    return __uint_as_float(i % 4 == 0 ? v.x : i % 4 == 1 ? v.y : i % 4 == 2 ? v.z : v.w);
  }
  __device__ __forceinline__ float magnitude() const {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, finite_magnitude(get(i)));
    return m;
  }
  __device__ __forceinline__ void store(uint8_t* p, float inverse) const {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      w[q] = f8_pack4(get(4 * q) * inverse, get(4 * q + 1) * inverse, get(4 * q + 2) * inverse, get(4 * q + 3) * inverse);
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Blocks of 1 x 128: block k of the [rows][nb] of them for every eight lanes.
template <int DTYPE>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantArgs a) {
  const int lane = threadIdx.x % 8;
  const int64_t blocks = a.rows * a.nb, step = (int64_t)gridDim.x * kRows;
  for (int64_t k = (int64_t)blockIdx.x * kRows + threadIdx.x / 8; k < blocks; k += step) {
    const int64_t row = k / a.nb;
    const int col = (int)(k % a.nb) * 128 + 16 * lane;
    const bool in = col < a.cols;
    Sixteen<DTYPE> x;
    if (in)
      x.load(a.X, row * a.cols + col);
    else
      x.clear();
    const int b = f8_scale(lanes_max<8>(x.magnitude()));
    if (in) x.store(a.X8 + row * a.cols + col, f8_inverse(b));
    if (lane == 0) a.scale[k] = (uint8_t)b;
  }
}

// Blocks of 128 x 128, a workgroup each.
template <int DTYPE>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(QuantArgs a) {
  constexpr int PASSES = 128 / kRows;
  __shared__ float side[2][4];
  int turn = 0;
  const int64_t blocks = (a.rows + 127) / 128 * a.nb;
  const int col_in = 16 * (threadIdx.x % 8), row_in = threadIdx.x / 8;
  for (int64_t k = blockIdx.x; k < blocks; k += gridDim.x) {
    const int64_t row0 = k / a.nb * 128;
    const int col = (int)(k % a.nb) * 128 + col_in;
    Sixteen<DTYPE> x[PASSES];
    float m = 0.f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int64_t row = row0 + p * kRows + row_in;
      if (row < a.rows && col < a.cols)
        x[p].load(a.X, row * a.cols + col);
      else
        x[p].clear();
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) m = fmaxf(m, x[p].magnitude());
    m = lanes_max<32>(m);
    m = fmaxf(m, __shfl_xor(m, 32));
    if (threadIdx.x % 64 == 0) side[turn][threadIdx.x / 64] = m;
    __syncthreads();  // (two sets in turn: one barrier a block is enough)
    m = fmaxf(fmaxf(side[turn][0], side[turn][1]), fmaxf(side[turn][2], side[turn][3]));
    turn ^= 1;
    const int b = f8_scale(m);
    const float inverse = f8_inverse(b);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int64_t row = row0 + p * kRows + row_in;
      if (row < a.rows && col < a.cols) x[p].store(a.X8 + row * a.cols + col, inverse);
    }
    if (threadIdx.x == 0) a.scale[k] = (uint8_t)b;
  }
}

template <int DTYPE>
bool launch(const QuantArgs& a, int rows_per_scale, hipStream_t s) {
  constexpr int64_t kMost = 1 << 20;  // workgroups of a launch; further blocks in further turns
  if (rows_per_scale == 1) {
    const int64_t grid = std::min((a.rows * a.nb + kRows - 1) / kRows, kMost);
    hipLaunchKernelGGL(quantize_rows_kernel<DTYPE>, dim3((unsigned)grid), dim3(256), 0, s, a);
  } else {
    const int64_t grid = std::min((a.rows + 127) / 128 * a.nb, kMost);
    hipLaunchKernelGGL(quantize_blocks_kernel<DTYPE>, dim3((unsigned)grid), dim3(256), 0, s, a);
  }
  return hipGetLastError() == hipSuccess;
}

}  // namespace

bool run_quantize(int dtype, const QuantArgs& a, int rows_per_scale, hipStream_t s) {
  return dtype == VP_BF16 ? launch<VP_BF16>(a, rows_per_scale, s) : launch<VP_F32>(a, rows_per_scale, s);
}

}  // namespace vpce
