// Losses of whole sequences behind the projection, for gfx950 (MI355X): a preference
// loss over pairs and a clipped policy loss with a KL term, with the gradient that the
// projection's backward takes.  The formulas are in vpce.h; everything between the
// float32 inputs and outputs is float64: a ratio next to a clip bound falls on the side
// it belongs to, e^q - q - 1 of a small q keeps its digits, and sums of any length are
// as good as one rounding of their result.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vpce_head.h"

namespace vpce {

namespace {

__device__ __forceinline__ int clip_offset(int v, int T) { return min(max(v, 0), T); }

// Tokens [lo, hi) of sequence s; false where its offsets are wrong.
__device__ __forceinline__ bool bounds(const SeqArgs& q, int s, int& lo, int& hi) {
  const int a = q.start[s], b = q.start[s + 1];
  lo = clip_offset(a, q.T);
  hi = clip_offset(b, q.T);
  return a == lo && b == hi && a <= b;
}

// The sequence of token t: the last one whose start is not behind it (S for tokens
// behind all of them, -1 for tokens before).  Any offsets end the search.
__device__ __forceinline__ int sequence_of(const SeqArgs& q, int t) {
  if (q.S == 0) return -1;
  int lo = -1, hi = q.S + 1;  // start[lo] <= t < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (q.start[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <int N>
__device__ void block_sum(double (&v)[N]) {
  __shared__ double part[N][4];
#pragma unroll
  for (int k = 0; k < N; ++k)
    for (int o = 32; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) part[k][threadIdx.x >> 6] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = (part[k][0] + part[k][1]) + (part[k][2] + part[k][3]);
}

// A preference pair from its two log ratio sums and token counts.
__device__ void finish_pair(const PrefArgs& a, int pair, const double (&sum)[2], const double (&n)[2],
                            bool good) {
  double c[2], reward[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    c[k] = !a.q.mean ? 1.0 : n[k] > 0.0 ? 1.0 / n[k] : 0.0;
    reward[k] = good ? a.beta * (c[k] * sum[k]) : __builtin_nan("");
  }
  const double z = reward[0] - reward[1] - a.margin;
  double loss, slope;
  if (a.kind == VP_PREF_LOGISTIC) {
    const double e = exp(-fabs(z)), l = log1p(e);
    const double pos = 1.0 / (1.0 + e), neg = e / (1.0 + e);  // sigmoid of |z| and of -|z|
    loss = (1.0 - a.smoothing) * (l + fmax(-z, 0.0));
    if (a.smoothing > 0.0) loss += a.smoothing * (l + fmax(z, 0.0));  // (an infinite z has weight 0 here)
    slope = a.smoothing * (z >= 0.0 ? pos : neg) - (1.0 - a.smoothing) * (z >= 0.0 ? neg : pos);
    if (!(z == z)) loss = z;
  } else {
    const double r = (z - 0.5) / a.beta;
    loss = r * r;
    slope = 2.0 * r / a.beta;
  }
  a.pair_loss[pair] = (float)loss;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    a.reward[2 * pair + k] = (float)reward[k];
    a.coef[2 * pair + k] = (float)((k ? slope : -slope) * a.beta * c[k]);
  }
}

__global__ void __launch_bounds__(256) pref_forward_kernel(PrefArgs a) {
  double sum[2], n[2];
  bool good = true;
  for (int k = 0; k < 2; ++k) {
    int lo, hi;
    good &= bounds(a.q, 2 * blockIdx.x + k, lo, hi);
    double v[2] = {0.0, 0.0};
    for (int t = lo + threadIdx.x; t < hi; t += 256)
      if (a.q.targets[t] != a.q.ignore_index) {
        v[0] += (a.ref ? (double)a.ref[t] : 0.0) - (double)a.loss[t];
        v[1] += 1.0;
      }
    block_sum(v);
    sum[k] = v[0];
    n[k] = v[1];
  }
  if (threadIdx.x == 0) finish_pair(a, blockIdx.x, sum, n, good);
}

__global__ void __launch_bounds__(256) pref_backward_kernel(SeqArgs q, const float* __restrict__ coef,
                                                            const float* __restrict__ grad_pair,
                                                            float* __restrict__ grad_loss) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= q.T) return;
  const int s = sequence_of(q, t);
  const bool counts = s >= 0 && s < q.S && q.targets[t] != q.ignore_index;
  grad_loss[t] = counts ? grad_pair[s >> 1] * coef[s] : 0.f;
}

// The policy loss of one token and its slope in loss_t.
struct PolicyToken {
  double loss, kl, slope;
  bool clipped;
};
__device__ __forceinline__ PolicyToken policy_token(const PolicyArgs& a, int t, double adv) {
  PolicyToken r;
  const double nll = (double)a.loss[t];
  // (a NaN loss makes x a NaN without an old loss, too)
  const double x = a.old ? (double)a.old[t] - nll : (nll == nll ? 0.0 : nll);
  r.clipped = adv > 0.0 ? x > a.log_high : adv < 0.0 ? x < a.log_low : false;
  const double rho = exp(x);
  // no advantage: 0 also where rho is infinite
  const double gain = adv == 0.0 ? (x == x ? 0.0 : x) : rho * adv;
  r.loss = r.clipped ? -((adv > 0.0 ? a.high : a.low) * adv) : -gain;
  r.slope = r.clipped ? 0.0 : gain;
  r.kl = 0.0;
  if (a.ref) {
    const double q = nll - (double)a.ref[t], em1 = expm1(q);
    r.kl = em1 == __builtin_inf() ? em1 : em1 - q;  // (q infinite: no difference of infinities)
    if (a.kl_coef > 0.0) {
      r.loss += a.kl_coef * r.kl;
      r.slope += a.kl_coef * em1;
    }
  }
  return r;
}

__global__ void __launch_bounds__(256) policy_forward_kernel(PolicyArgs a) {
  const int s = blockIdx.x;
  int lo, hi;
  const bool good = bounds(a.q, s, lo, hi);
  double v[4] = {0.0, 0.0, 0.0, 0.0};
  for (int t = lo + threadIdx.x; t < hi; t += 256)
    if (a.q.targets[t] != a.q.ignore_index) {
      const PolicyToken r = policy_token(a, t, (double)a.adv[a.per_token ? t : s]);
      v[0] += r.loss;
      v[1] += r.kl;
      v[2] += r.clipped ? 1.0 : 0.0;
      v[3] += 1.0;
    }
  block_sum(v);
  if (threadIdx.x == 0) {
    const double c = !good ? __builtin_nan("") : !a.q.mean ? 1.0 : v[3] > 0.0 ? 1.0 / v[3] : 0.0;
    a.seq_loss[s] = (float)(c * v[0]);
    a.seq_kl[s] = (float)(c * v[1]);
    a.clipped[s] = good ? (int)v[2] : 0;
    a.tokens[s] = good ? (int)v[3] : 0;
  }
}

__global__ void __launch_bounds__(256) policy_backward_kernel(PolicyArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= a.q.T) return;
  const int s = sequence_of(a.q, t);
  float g = 0.f;
  if (s >= 0 && s < a.q.S && a.q.targets[t] != a.q.ignore_index) {
    const double c = a.q.mean ? 1.0 / (double)max(a.tokens[s], 1) : 1.0;
    g = (float)((double)a.grad_seq[s] * c * policy_token(a, t, (double)a.adv[a.per_token ? t : s]).slope);
  }
  a.grad_loss[t] = g;
}

bool launched_ok() { return hipGetLastError() == hipSuccess; }
unsigned blocks(int n) { return (unsigned)((n + 255) / 256); }

}  // namespace

bool run_pref_forward(const PrefArgs& a, hipStream_t s) {
  if (a.q.S == 0) return true;
  hipLaunchKernelGGL(pref_forward_kernel, dim3((unsigned)a.q.S / 2), dim3(256), 0, s, a);
  return launched_ok();
}
bool run_pref_backward(const SeqArgs& q, const float* coef, const float* grad_pair, float* grad_loss,
                       hipStream_t s) {
  if (q.T == 0) return true;
  hipLaunchKernelGGL(pref_backward_kernel, dim3(blocks(q.T)), dim3(256), 0, s, q, coef, grad_pair, grad_loss);
  return launched_ok();
}
bool run_policy_forward(const PolicyArgs& a, hipStream_t s) {
  if (a.q.S == 0) return true;
  hipLaunchKernelGGL(policy_forward_kernel, dim3((unsigned)a.q.S), dim3(256), 0, s, a);
  return launched_ok();
}
bool run_policy_backward(const PolicyArgs& a, hipStream_t s) {
  if (a.q.T == 0) return true;
  hipLaunchKernelGGL(policy_backward_kernel, dim3(blocks(a.q.T)), dim3(256), 0, s, a);
  return launched_ok();
}

}  // namespace vpce
