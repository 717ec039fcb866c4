// Layer norm of the hidden states and its gradients, for gfx950 (MI355X).  Memory
// bound: the forward reads X and writes Y, the backward reads X and dY and writes dX.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vpce_head.h"

namespace vpce {

namespace {

struct Half {  // bfloat16
  using storage = uint16_t;
  __device__ static float load(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
  // round to nearest even; a NaN stays a NaN
  __device__ static uint16_t store(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
};
struct Single {
  using storage = float;
  __device__ static float load(float f) { return f; }
  __device__ static float store(float f) { return f; }
};

// Sum over a workgroup of 256 threads, the same bits in every thread.
__device__ float block_sum(float v) {
  __shared__ float part[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <class E, bool RMS>
__global__ void __launch_bounds__(256) norm_forward_kernel(NormArgs a) {
  using S = typename E::storage;
  const int64_t t = blockIdx.x;
  const S* x = (const S*)a.X + t * a.d;
  float mean = 0.f;
  if (!RMS) {
    float sum = 0.f;
    for (int j = threadIdx.x; j < a.d; j += 256) sum += E::load(x[j]);
    mean = block_sum(sum) / (float)a.d;
  }
  float sq = 0.f;
  for (int j = threadIdx.x; j < a.d; j += 256) {
    const float v = E::load(x[j]) - mean;
    sq += v * v;
  }
  const float rstd = 1.f / sqrtf(block_sum(sq) / (float)a.d + a.eps);
  for (int j = threadIdx.x; j < a.d; j += 256) {
    float y = (E::load(x[j]) - mean) * rstd * E::load(((const S*)a.gamma)[j]);
    if (a.beta) y += E::load(((const S*)a.beta)[j]);
    ((S*)a.Y)[t * a.d + j] = E::store(y);
  }
  if (threadIdx.x == 0) {
    a.rstd[t] = rstd;
    if (!RMS) a.mean[t] = mean;
  }
}

// dgamma and dbeta first (dX may overwrite dY): one thread a column.
template <class E, bool RMS>
__global__ void __launch_bounds__(64) norm_weight_grad_kernel(NormGradArgs a) {
  using S = typename E::storage;
  const int j = blockIdx.x * 64 + threadIdx.x;
  if (j >= a.d) return;
  float dg = 0.f, db = 0.f;
  for (int64_t t = 0; t < a.T; ++t) {
    const float dy = a.dY[t * a.d + j];
    const float mean = RMS ? 0.f : a.mean[t];
    dg += dy * ((E::load(((const S*)a.X)[t * a.d + j]) - mean) * a.rstd[t]);
    db += dy;
  }
  a.dgamma[j] = a.accumulate ? a.dgamma[j] + dg : dg;
  if (a.dbeta) a.dbeta[j] = a.accumulate ? a.dbeta[j] + db : db;
}

template <class E, bool RMS>
__global__ void __launch_bounds__(256) norm_input_grad_kernel(NormGradArgs a) {
  using S = typename E::storage;
  const int64_t t = blockIdx.x;
  const S* x = (const S*)a.X + t * a.d;
  const float mean = RMS ? 0.f : a.mean[t], rstd = a.rstd[t];
  float s1 = 0.f, s2 = 0.f;
  for (int j = threadIdx.x; j < a.d; j += 256) {
    const float g = a.dY[t * a.d + j] * E::load(((const S*)a.gamma)[j]);
    s1 += g;
    s2 += g * ((E::load(x[j]) - mean) * rstd);
  }
  const float c1 = RMS ? 0.f : block_sum(s1) / (float)a.d;
  const float c2 = block_sum(s2) / (float)a.d;
  for (int j = threadIdx.x; j < a.d; j += 256) {
    const float g = a.dY[t * a.d + j] * E::load(((const S*)a.gamma)[j]);
    a.dX[t * a.d + j] = rstd * (g - c1 - (E::load(x[j]) - mean) * rstd * c2);
  }
}

bool launched_ok() { return hipGetLastError() == hipSuccess; }

template <class E, bool RMS>
bool forward(const NormArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((norm_forward_kernel<E, RMS>), dim3((unsigned)a.T), dim3(256), 0, s, a);
  return launched_ok();
}
template <class E, bool RMS>
bool backward(const NormGradArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((norm_weight_grad_kernel<E, RMS>), dim3((unsigned)((a.d + 63) / 64)), dim3(64), 0, s, a);
  if (!launched_ok()) return false;
  if (a.T == 0) return true;
  hipLaunchKernelGGL((norm_input_grad_kernel<E, RMS>), dim3((unsigned)a.T), dim3(256), 0, s, a);
  return launched_ok();
}

}  // namespace

bool run_norm_forward(int dtype, bool rms, const NormArgs& a, hipStream_t s) {
  if (dtype == VP_BF16) return rms ? forward<Half, true>(a, s) : forward<Half, false>(a, s);
  return rms ? forward<Single, true>(a, s) : forward<Single, false>(a, s);
}
bool run_norm_backward(int dtype, bool rms, const NormGradArgs& a, hipStream_t s) {
  if (dtype == VP_BF16) return rms ? backward<Half, true>(a, s) : backward<Half, false>(a, s);
  return rms ? backward<Single, true>(a, s) : backward<Single, false>(a, s);
}

}  // namespace vpce
