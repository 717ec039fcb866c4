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

constexpr int kRound = 256;  // tokens that a wavefront takes at a time, four a lane

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }

template <int N>
__device__ __forceinline__ void wave_sum(double (&v)[N]) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], o);
}

// The sequence of token t: the last one whose start is not behind it, S for tokens
// behind all of them, -1 for tokens before.  One wavefront, 64 probes at a time; for any
// offsets it ends and the answer is in -1..S.
__device__ __forceinline__ int sequence_of(const SeqArgs& q, int t) {
  if (q.S == 0) return -1;
  int lo = 0, n = q.S + 1;  // start[i] <= t for i < lo, start[i] > t for i >= lo + n
  while (n > 64) {
    const int step = (n + 63) / 64, i = lo + (lane_id() + 1) * step - 1;
    const int c = __popcll(__ballot(i < lo + n && q.start[min(i, q.S)] <= t));
    lo += c * step;
    n = min(step - 1, n - c * step);
  }
  const int i = lo + lane_id();
  return lo + __popcll(__ballot(lane_id() < n && q.start[min(i, q.S)] <= t)) - 1;
}

// The sequences of up to 64 tokens in order, one a lane, the first of them at or behind
// sequence s: counts the offsets behind start[s] that are not behind the lane's token.
// `last` is the last lane's token.  For any offsets it ends and the answer is in s..S.
__device__ __forceinline__ int sequences_from(const SeqArgs& q, int s, int t, int last) {
  int mine = s;
  for (int first = s + 1; first <= q.S; first += 64) {
    const int i = first + lane_id();
    const int o = i <= q.S ? q.start[i] : INT32_MAX;
    int lo = 0, hi = 64;  // o of lanes < lo is not behind t, o of lanes >= hi is
#pragma unroll
    for (int k = 0; k < 7; ++k) {
      const int mid = (lo + hi) >> 1, at = __shfl(o, mid & 63);
      if (lo < hi) {
        if (at <= t)
          lo = mid + 1;
        else
          hi = mid;
      }
    }
    mine += lo;
    if (__shfl(o, 63) > last) break;
  }
  return mine;
}

// End of sequence s: its tokens are in front of it (tokens before the first: s = -1).
__device__ __forceinline__ int end_of(const SeqArgs& q, int s) { return s < q.S ? q.start[s + 1] : INT32_MAX; }

// Partial sums.  The tokens are cut into chunks of q.chunk, a wavefront each, and chunk c
// leaves its part of sequence s in slot c + s: walking the tokens, every step to another
// chunk or sequence makes c + s larger, so no two parts share a slot, and chunks + S slots
// are enough.
//
// The sums of the sequence that a chunk is in stay spread over the lanes as long as it
// lasts.  Where a round of tokens holds an end, its tokens go through a segmented scan, 64
// at a time, which takes the same time for one end or 63.
template <class Op>
__device__ __forceinline__ void chunk_sums(const Op& op, int c) {
  constexpr int K = Op::K;
  const SeqArgs& q = op.a.q;
  const int lane = lane_id();
  const int t0 = c * q.chunk, t1 = min(q.T, t0 + q.chunk);
  if (t0 >= t1) return;
  double* part = q.part;
  auto put = [&](int s, const double (&v)[K]) {
    if (s < 0 || s >= q.S) return;
#pragma unroll
    for (int k = 0; k < K; ++k) part[(int64_t)(c + s) * K + k] = v[k];
  };
  double acc[K];
#pragma unroll
  for (int k = 0; k < K; ++k) acc[k] = 0.0;
  int s = -2, end = 0;  // the sequence that the walk is in, and its end
  for (int base = t0; base < t1; base += kRound) {
    typename Op::Raw raw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) op.load(raw[j], min(base + 64 * j + lane, t1 - 1));
    if (s == -2) {  // (behind the first loads)
      s = sequence_of(q, t0);
      end = end_of(q, s);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int b = base + 64 * j, e = min(b + 64, t1);
      if (b >= t1) break;
      const bool in = b + lane < e;
      if (e <= end) {
        if (in && s >= 0 && s < q.S) op.add(acc, raw[j], s);
        continue;
      }
      // an end inside: close the lanes' sums and scan
      wave_sum(acc);
      const int mine = sequences_from(q, s, min(b + lane, e - 1), e - 1);
      double v[K];
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = 0.0;
      if (in && mine >= 0 && mine < q.S) op.add(v, raw[j], mine);
      const int up = __shfl_up(mine, 1), next = __shfl_down(mine, 1);  // (every lane takes part)
      bool head = mine != (lane ? up : s);
      if (lane == 0) {
        if (head)
          put(s, acc);
        else
#pragma unroll
          for (int k = 0; k < K; ++k) v[k] += acc[k];
      }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const bool h = __shfl_up((int)head, o);
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const double w = __shfl_up(v[k], o);
          if (lane >= o && !head) v[k] += w;
        }
        if (lane >= o) head |= h;
      }
      if (lane < 63 && next != mine) put(mine, v);
      // the last lane's sequence goes on
      s = __shfl(mine, 63);
      end = end_of(q, s);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const double w = __shfl(v[k], 63);
        acc[k] = lane ? 0.0 : w;
      }
    }
  }
  wave_sum(acc);
  if (lane == 0) put(s, acc);
}

// Sums of sequence s over its chunks, LANES lanes side by side; false where its offsets
// are wrong.
template <int K, int LANES>
__device__ __forceinline__ bool sequence_sums(const SeqArgs& q, int s, double (&v)[K]) {
  const int a = q.start[s], b = q.start[s + 1];
  const bool good = 0 <= a && a <= b && b <= q.T;
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.0;
  if (good && a < b) {
    const int last = (b - 1) / q.chunk;
#pragma unroll 2
    for (int c = a / q.chunk + (int)(threadIdx.x % LANES); c <= last; c += LANES)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += q.part[(int64_t)(c + s) * K + k];
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o);
  return good;
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

struct PrefOp {
  static constexpr int K = 2;  // log ratios, counting tokens
  struct Raw {
    int64_t target;
    float loss, ref;
  };
  const PrefArgs& a;
  __device__ __forceinline__ void load(Raw& r, int t) const {
    r.target = a.q.targets[t];
    r.loss = a.loss[t];
    r.ref = a.ref ? a.ref[t] : 0.f;
  }
  __device__ __forceinline__ void add(double (&v)[K], const Raw& r, int) const {
    if (r.target == a.q.ignore_index) return;
    v[0] += (double)r.ref - (double)r.loss;
    v[1] += 1.0;
  }
  static constexpr int PER_UNIT = 2;  // a unit is a pair
  template <int LANES>
  __device__ __forceinline__ void finish(int pair) const {
    double v[2][K], sum[2], n[2];
    bool good = true;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      good &= sequence_sums<K, LANES>(a.q, 2 * pair + k, v[k]);
      sum[k] = v[k][0];
      n[k] = v[k][1];
    }
    if (threadIdx.x % LANES == 0) finish_pair(a, pair, sum, n, good);
  }
};

// The policy loss of one token and its slope in loss_t.
struct PolicyToken {
  double loss, kl, slope;
  bool clipped;
};
struct PolicyRaw {
  int64_t target;
  float loss, old, ref, adv;
};
__device__ __forceinline__ void load_token(const PolicyArgs& a, PolicyRaw& r, int t) {
  r.target = a.q.targets[t];
  r.loss = a.loss[t];
  r.old = a.old ? a.old[t] : 0.f;
  r.ref = a.ref ? a.ref[t] : 0.f;
  r.adv = a.per_token ? a.adv[t] : 0.f;
}
__device__ __forceinline__ PolicyToken policy_token(const PolicyArgs& a, const PolicyRaw& t, double adv) {
  PolicyToken r;
  const double nll = (double)t.loss;
  // (a NaN loss makes x a NaN without an old loss, too)
  const double x = a.old ? (double)t.old - nll : (nll == nll ? 0.0 : nll);
  r.clipped = adv > 0.0 ? x > a.log_high : adv < 0.0 ? x < a.log_low : false;
  const double rho = a.old ? exp(x) : 1.0 + x;
  // no advantage: 0 also where rho is infinite
  const double gain = adv == 0.0 ? (x == x ? 0.0 : x) : rho * adv;
  r.loss = r.clipped ? -((adv > 0.0 ? a.high : a.low) * adv) : -gain;
  r.slope = r.clipped ? 0.0 : gain;
  r.kl = 0.0;
  if (a.ref) {
    const double q = nll - (double)t.ref, em1 = expm1(q);
    r.kl = em1 == __builtin_inf() ? em1 : em1 - q;  // (q infinite: no difference of infinities)
    if (a.kl_coef > 0.0) {
      r.loss += a.kl_coef * r.kl;
      r.slope += a.kl_coef * em1;
    }
  }
  return r;
}

struct PolicyOp {
  // losses, KL terms, and both counts in one: clipped tokens times 2^23 (there are fewer
  // tokens than that) plus counting tokens, whole numbers below 2^46
  static constexpr int K = 3;
  static constexpr double kClip = 8388608.0;
  using Raw = PolicyRaw;
  const PolicyArgs& a;
  __device__ __forceinline__ void load(Raw& r, int t) const { load_token(a, r, t); }
  __device__ __forceinline__ void add(double (&v)[K], const Raw& r, int s) const {
    if (r.target == a.q.ignore_index) return;
    const PolicyToken p = policy_token(a, r, (double)(a.per_token ? r.adv : a.adv[s]));
    v[0] += p.loss;
    v[1] += p.kl;
    v[2] += p.clipped ? kClip + 1.0 : 1.0;
  }
  static constexpr int PER_UNIT = 1;  // a unit is a sequence
  template <int LANES>
  __device__ __forceinline__ void finish(int s) const {
    double v[K];
    const bool good = sequence_sums<K, LANES>(a.q, s, v);
    if (threadIdx.x % LANES) return;
    const double clipped = floor(v[2] / kClip), n = v[2] - clipped * kClip;
    const double c = !good ? __builtin_nan("") : !a.q.mean ? 1.0 : n > 0.0 ? 1.0 / n : 0.0;
    a.seq_loss[s] = (float)(c * v[0]);
    a.seq_kl[s] = (float)(c * v[1]);
    a.clipped[s] = (int)clipped;
    a.tokens[s] = (int)n;
  }
};

template <class Op, class Args>
__global__ void __launch_bounds__(256) chunk_kernel(Args args) {
  const Op op{args};
  chunk_sums(op, __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)));
}
template <class Op, class Args, int LANES>
__global__ void __launch_bounds__(256) finish_kernel(Args args) {
  const Op op{args};
  const int unit = (blockIdx.x * 256 + threadIdx.x) / LANES;
  if (unit < args.q.S / Op::PER_UNIT) op.template finish<LANES>(unit);
}
// Both in one launch, for tokens that one workgroup holds.
template <class Op, class Args>
__global__ void __launch_bounds__(1024) small_kernel(Args args) {
  const Op op{args};
  chunk_sums(op, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  __syncthreads();
  for (int unit = threadIdx.x; unit < args.q.S / Op::PER_UNIT; unit += 1024) op.template finish<1>(unit);
}

// Gradients: a round of tokens a wavefront.
struct PrefGrad {
  SeqArgs q;
  const float* coef;
  const float* grad_pair;
  float* grad_loss;
  struct Raw {
    int64_t target;
  };
  __device__ __forceinline__ void load(Raw& r, int t) const { r.target = q.targets[t]; }
  __device__ __forceinline__ float grad(const Raw&, int s) const { return grad_pair[s >> 1] * coef[s]; }
};
struct PolicyGrad {
  PolicyArgs a;
  SeqArgs q;
  float* grad_loss;
  using Raw = PolicyRaw;
  __device__ __forceinline__ void load(Raw& r, int t) const { load_token(a, r, t); }
  __device__ __forceinline__ float grad(const Raw& r, int s) const {
    const double c = q.mean ? 1.0 / (double)max(a.tokens[s], 1) : 1.0;
    return (float)((double)a.grad_seq[s] * c *
                   policy_token(a, r, (double)(a.per_token ? r.adv : a.adv[s])).slope);
  }
};
template <class Op>
__global__ void __launch_bounds__(256) grad_kernel(Op op) {
  const SeqArgs& q = op.q;
  const int lane = lane_id();
  const int base = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)) * kRound;
  if (base >= q.T) return;
  typename Op::Raw raw[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) op.load(raw[j], min(base + 64 * j + lane, q.T - 1));
  int s = sequence_of(q, base), end = end_of(q, s);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int b = base + 64 * j, e = min(b + 64, q.T);
    if (b >= q.T) break;
    int mine = s;
    if (e > end) {
      mine = sequences_from(q, s, min(b + lane, e - 1), e - 1);
      s = __shfl(mine, 63);
      end = end_of(q, s);
    }
    if (b + lane < e) {
      const bool counts = mine >= 0 && mine < q.S && raw[j].target != q.ignore_index;
      op.grad_loss[b + lane] = counts ? op.grad(raw[j], mine) : 0.f;
    }
  }
}

bool launched_ok() { return hipGetLastError() == hipSuccess; }

template <class Op, class Args>
bool forward(const Args& a, hipStream_t s) {
  const SeqArgs& q = a.q;
  if (q.S == 0) return true;
  const SeqPlan p = seq_plan(q.T, q.S);
  if (p.chunks <= 16) {
    hipLaunchKernelGGL((small_kernel<Op, Args>), dim3(1), dim3(1024), 0, s, a);
    return launched_ok();
  }
  hipLaunchKernelGGL((chunk_kernel<Op, Args>), dim3((unsigned)(p.chunks + 3) / 4), dim3(256), 0, s, a);
  if (!launched_ok()) return false;
  const int units = q.S / Op::PER_UNIT;
  if (units <= 16384)
    hipLaunchKernelGGL((finish_kernel<Op, Args, 64>), dim3((unsigned)(units + 3) / 4), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((finish_kernel<Op, Args, 8>), dim3((unsigned)(units + 31) / 32), dim3(256), 0, s, a);
  return launched_ok();
}
template <class Op>
bool backward(const Op& op, hipStream_t s) {
  if (op.q.T == 0) return true;
  const unsigned rounds = (unsigned)(op.q.T + kRound - 1) / kRound;
  hipLaunchKernelGGL((grad_kernel<Op>), dim3((rounds + 3) / 4), dim3(256), 0, s, op);
  return launched_ok();
}

}  // namespace

SeqPlan seq_plan(int T, int S) {
  SeqPlan p;
  const int rounds = (T + kRound - 1) / kRound;
  p.chunk = kRound * ((rounds + 4095) / 4096 > 0 ? (rounds + 4095) / 4096 : 1);
  p.chunks = (T + p.chunk - 1) / p.chunk;
  p.slots = (int64_t)p.chunks + S;
  return p;
}

bool run_pref_forward(const PrefArgs& a, hipStream_t s) { return forward<PrefOp>(a, s); }
bool run_pref_backward(const SeqArgs& q, const float* coef, const float* grad_pair, float* grad_loss,
                       hipStream_t s) {
  return backward(PrefGrad{q, coef, grad_pair, grad_loss}, s);
}
bool run_policy_forward(const PolicyArgs& a, hipStream_t s) { return forward<PolicyOp>(a, s); }
bool run_policy_backward(const PolicyArgs& a, hipStream_t s) {
  return backward(PolicyGrad{a, a.q, a.grad_loss}, s);
}

}  // namespace vpce
