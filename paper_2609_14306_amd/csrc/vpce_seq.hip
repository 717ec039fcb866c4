// Losses of whole sequences behind the projection, for gfx950 (MI355X): a preference
// loss over pairs and a clipped policy loss with a KL term, with the gradient that the
// projection's backward takes.  The formulas are in vpce.h; everything between the
// float32 inputs and outputs is float64: a ratio next to a clip bound falls on the side
// it belongs to, e^q - q - 1 of a small q keeps its digits, and sums of any length are
// as good as one rounding of their result.
//
// Bound: up to some 100000 tokens by launches and by the latency of a few dependent loads
// (offsets, a sequence's values, partial sums); beyond by memory, 16 to 24 bytes a token in
// the forward and 12 to 28 in the backward, and in the policy forward as much by its float64
// arithmetic (171 vector instructions for 64 tokens).  MI355X, kernels alone, averages: T = 32768
// in 64 sequences, policy 4.9 + 2.9 us forward, 3.8 us backward; T = 4.2 M in 4096, 29.6 + 4.7 us
// (3.4 TB/s) and 22.8 us (5.1 TB/s); preference, T = 4.0 M in 2500 pairs, 16.1 + 4.1 us
// (4.0 TB/s) and 11.1 us (4.3 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "vpce_head.h"
#include "vpce_lanes.h"

namespace vpce {

namespace {

// Wavefronts that the tokens are spread over, 64 tokens at a time each: rounds of 64 leave
// few tokens to the scans, and enough of them hide each other's loads and arithmetic (4.2 M
// tokens, policy forward: 16384 wavefronts 30.6 us, 4096 with four loads on their way 33.1).
constexpr int kWaves = 16384;

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }

// Sum over a wavefront, the same in every lane.
template <int N>
__device__ __forceinline__ void wave_sum(double (&v)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] += lane_move<kSwap1>(v[k]);
    v[k] += lane_move<kSwap2>(v[k]);
    v[k] += lane_move<kHalfMirror>(v[k]);
    v[k] += lane_move<kMirror>(v[k]);
    v[k] = (lane_read(v[k], 0) + lane_read(v[k], 16)) + (lane_read(v[k], 32) + lane_read(v[k], 48));
  }
}

// Sums over the lanes from the last head at or in front of each lane up to it.
template <int CTRL, int ROWS, int N>
__device__ __forceinline__ void scan_step(double (&v)[N], int& head) {
  const int h = lane_move<CTRL, ROWS>(head);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const double w = lane_move<CTRL, ROWS>(v[k]);
    v[k] = head ? v[k] : v[k] + w;
  }
  head |= h;
}
template <int N>
__device__ __forceinline__ void segmented_scan(double (&v)[N], int head) {
  scan_step<kUp1, 0xf>(v, head);
  scan_step<kUp2, 0xf>(v, head);
  scan_step<kUp4, 0xf>(v, head);
  scan_step<kUp8, 0xf>(v, head);
  scan_step<kRowEnd, 0xa>(v, head);
  scan_step<kHalfEnd, 0xc>(v, head);
}

// 64 consecutive offsets, one a lane: start[base + lane] (INT32_MAX behind the last).
// The sequence of a token t is the last one whose start is not behind it, S for tokens
// behind all of them and -1 for tokens before.  Whatever the offsets are, every walk
// below ends and every sequence it names is in -1..S.
struct Window {
  int base, o;
  __device__ __forceinline__ void load(const SeqArgs& q) {
    o = base + lane_id() <= q.S && q.S > 0 ? q.start[base + lane_id()] : INT32_MAX;
  }
  // Moves to where token t is, 64 probes at a time; its sequence.
  __device__ __forceinline__ int open(const SeqArgs& q, int t) {
    int lo = 0, n = q.S + 1;  // start[i] <= t for i < lo, start[i] > t for i >= lo + n
    while (n > 64) {
      const int step = (n + 63) / 64, i = lo + (lane_id() + 1) * step - 1;
      const int c = __popcll(__ballot(i < lo + n && q.start[min(i, q.S)] <= t));
      lo += c * step;
      n = min(step - 1, n - c * step);
    }
    base = lo;
    load(q);
    return base - 1 + __popcll(__ballot(o <= t));
  }
  // End of sequence s, the last one looked up.
  __device__ __forceinline__ int end(const SeqArgs& q, int s) const {
    const int i = s + 1 - base;
    if (i >= 0 && i < 64) return __builtin_amdgcn_readlane(o, i);
    return s < q.S ? q.start[s + 1] : INT32_MAX;
  }
  // Sequences of the tokens first..last, one a lane (the lanes behind get last's), which
  // are not in front of a token looked up before.
  __device__ __forceinline__ int walk(const SeqArgs& q, int first, int last) {
    const int t = min(first + lane_id(), last);
    int s = base - 1;
    for (;;) {
      s += __popcll(__ballot(o <= first));
      for (uint64_t m = __ballot(o > first && o <= last); m; m &= m - 1)
        s += __builtin_amdgcn_readlane(o, __builtin_ctzll(m)) <= t;
      const int v = __builtin_amdgcn_readlane(o, 63);
      if (v > last) return s;
      base += 64;
      // A window of one offset: a run of empty sequences.  It is left by the largest step of
      // 64, 128, 256, ... that stays in it (4 M of them inside 64 tokens, a call: 0.2 ms instead
      // of the 199 of a window at a time).
      if (__builtin_amdgcn_readlane(o, 0) == v) {
        const int i = base + (64 << min(lane_id(), 16));
        const int c = __popcll(__ballot(i <= q.S && q.start[min(i, q.S)] <= v));
        if (c > 0) {
          base += 32 << c;
          s = t < v ? s : base - 1;
        }
      }
      load(q);
    }
  }
};

// A sequence that exists in place of -1 and S, whose values are read and not used.
__device__ __forceinline__ int clip(int s, const SeqArgs& q) { return min(max(s, 0), max(q.S - 1, 0)); }

// Partial sums.  The tokens are cut into chunks of q.chunk, a wavefront each, and chunk c
// leaves its part of sequence s in slot c + s: walking the tokens, every step to another
// chunk or sequence makes c + s larger, so no two parts share a slot, and chunks + S slots
// are enough.
//
// The sums of the sequence that a chunk is in stay spread over the lanes as long as it
// lasts.  64 tokens that hold an end go through a segmented scan, which takes the same
// time for one end or 63.  The next 64 tokens are on their way meanwhile.
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
  typename Op::Raw raw, next;
  op.load(next, min(t0 + lane, t1 - 1));
  Window w;
  int s = w.open(q, t0), end = w.end(q, s);  // the sequence that the walk is in, and its end
  typename Op::Seq here = op.open(clip(s, q));
  for (int b = t0; b < t1; b += 64) {
    const int e = min(b + 64, t1);
    raw = next;
    op.load(next, min(e + lane, t1 - 1));
    const bool cut = e > end;
    const int mine = cut ? w.walk(q, b, e - 1) : s;
    double v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.0;
    typename Op::Seq seq = here;
    if (cut) {
      seq = op.open(clip(mine, q));
      seq.wait();  // here, where there is something to wait for
    }
    if (b + lane < e && mine >= 0 && mine < q.S) op.add(v, raw, seq);
    if (!cut) {
#pragma unroll
      for (int k = 0; k < K; ++k) acc[k] += v[k];
      continue;
    }
    wave_sum(acc);
    const int up = __shfl_up(mine, 1), down = __shfl_down(mine, 1);
    const bool head = mine != (lane ? up : s);
    if (lane == 0) {
      if (head)
        put(s, acc);
      else
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += acc[k];
    }
    segmented_scan(v, (int)head);
    if (lane < 63 && down != mine) put(mine, v);
    // the last lane's sequence goes on
    s = __builtin_amdgcn_readlane(mine, 63);
    end = w.end(q, s);
    here = op.open(clip(s, q));
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const double x = lane_read(v[k], 63);
      acc[k] = lane ? 0.0 : x;
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
#pragma unroll 8
    for (int c = a / q.chunk + (int)(threadIdx.x % LANES); c <= last; c += LANES)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += q.part[(int64_t)(c + s) * K + k];
  }
  if constexpr (LANES >= 64) {
    wave_sum(v);
  } else {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o);
  }
  if constexpr (LANES > 64) {  // a workgroup of 256, or its halves
    __shared__ double side[4][K];
    const int first = threadIdx.x / LANES * (LANES / 64);
    if (lane_id() == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) side[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = side[first][k];
#pragma unroll
      for (int w = 1; w < LANES / 64; ++w) v[k] += side[first + w][k];
    }
  }
  return good;
}

// e^x, e^x - 1 and e^x - 1 - x: x = n ln 2 + r with |r| <= 0.3466, p = e^r - 1 = r + tail by its
// series up to r^11 / 11! (what is left out is below 2^-45 r and 2^-42 of the tail), e^x =
// 2^n (1 + p).  For n = 0 the other two are p and the tail themselves, so a small x keeps the
// digits of its x^2 / 2; otherwise each loses at most five bits to its difference (|x| >= 0.3466:
// e^x - 1 - x >= 0.05).  Fewer instructions than the math library's exp and expm1, which carry
// their answers to the last bit of a double.
__device__ __forceinline__ void exp_both(double x, double& e, double& em1, double& rest) {
  const double y = fmin(fmax(x, -1100.0), 1100.0);
  const double n = rint(y * 1.4426950408889634);
  double r = fma(n, -0.6931471805599453, y);
  r = fma(n, -2.3190468138462996e-17, r);
  double p = 1.0 / 39916800.0;
  p = fma(p, r, 1.0 / 3628800.0);
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  const double half = p * r, tail = half * r;
  p = fma(half, r, r);
  e = ldexp(1.0 + p, (int)n);
  em1 = n == 0.0 ? p : e - 1.0;
  rest = n == 0.0 ? tail : em1 == __builtin_inf() ? em1 : em1 - x;  // (no difference of infinities)
  if (!(x == x)) e = em1 = rest = x;
}

// log(1 + e) for 0 <= e <= 1: 2 atanh(u), u = e / (2 + e) <= 1/3, by its series up to
// u^29 / 29 (the next term is below 2^-51 u).
__device__ __forceinline__ double log_1_plus(double e) {
  const double u = e / (2.0 + e), w = u * u;
  double p = 1.0 / 29.0;
#pragma unroll
  for (int k = 27; k >= 1; k -= 2) p = fma(p, w, 1.0 / k);
  return 2.0 * u * p;
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
    double e, unused[2];
    exp_both(-fabs(z), e, unused[0], unused[1]);
    const double l = log_1_plus(e);
    const double pos = 1.0 / (1.0 + e), neg = e * pos;  // sigmoid of |z| and of -|z|
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
    r.ref = a.ref[t];
  }
  struct Seq {
    __device__ void wait() {}
  };
  __device__ __forceinline__ Seq open(int) const { return {}; }
  __device__ __forceinline__ void add(double (&v)[K], const Raw& r, const Seq&) const {
    if (r.target == a.q.ignore_index) return;
    v[0] += (a.has_ref ? (double)r.ref : 0.0) - (double)r.loss;
    v[1] += 1.0;
  }
  static constexpr int PER_UNIT = 2;  // a unit is a pair, its sequences side by side
  template <int LANES>
  __device__ __forceinline__ void finish(int pair) const {
    constexpr int H = LANES / 2;
    const int half = threadIdx.x / H & 1;
    double v[K], sum[2], n[2];
    bool good = sequence_sums<K, H>(a.q, 2 * pair + half, v);
    if constexpr (LANES > 64) {
      __shared__ double both[2][K];
      __shared__ int fine[2];
      if (threadIdx.x % H == 0) {
        both[half][0] = v[0];
        both[half][1] = v[1];
        fine[half] = good;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        sum[k] = both[k][0];
        n[k] = both[k][1];
      }
      good = fine[0] && fine[1];
    } else {
      const double s1 = __shfl_xor(v[0], H), n1 = __shfl_xor(v[1], H);
      good = (int)good & __shfl_xor((int)good, H);
      sum[0] = v[0], sum[1] = s1;  // (as the first half needs them)
      n[0] = v[1], n[1] = n1;
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
  r.old = a.old[t];
  r.ref = a.ref[t];
  r.adv = a.adv_tok[t];
}
__device__ __forceinline__ PolicyToken policy_token(const PolicyArgs& a, const PolicyRaw& t, double adv) {
  PolicyToken r;
  const double nll = (double)t.loss;
  // (a NaN loss makes x a NaN without an old loss, too)
  const double x = a.has_old ? (double)t.old - nll : (nll == nll ? 0.0 : nll);
  r.clipped = adv > 0.0 ? x > a.log_high : adv < 0.0 ? x < a.log_low : false;
  double rho = 1.0 + x, unused[2];
  if (a.has_old) exp_both(x, rho, unused[0], unused[1]);
  // no advantage: 0 also where rho is infinite
  const double gain = adv == 0.0 ? (x == x ? 0.0 : x) : rho * adv;
  r.loss = r.clipped ? -((adv > 0.0 ? a.high : a.low) * adv) : -gain;
  r.slope = r.clipped ? 0.0 : gain;
  r.kl = 0.0;
  if (a.has_ref) {
    double em1;
    exp_both(nll - (double)t.ref, unused[0], em1, r.kl);
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
  struct Seq {
    float adv;
    __device__ __forceinline__ void wait() { asm volatile("" : "+v"(adv)); }
  };
  __device__ __forceinline__ Seq open(int s) const { return {a.per_token ? 0.f : a.adv[s]}; }
  __device__ __forceinline__ void add(double (&v)[K], const Raw& r, const Seq& seq) const {
    if (r.target == a.q.ignore_index) return;
    const PolicyToken p = policy_token(a, r, (double)(a.per_token ? r.adv : seq.adv));
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
  constexpr int LANES = Op::PER_UNIT;
  for (int unit = threadIdx.x / LANES; unit < args.q.S / Op::PER_UNIT; unit += 1024 / LANES)
    op.template finish<LANES>(unit);
}

// Gradients: J tokens a lane, one where more would not fill the chip (4 M tokens, J = 1 / 2 /
// 4: preference 16.8 / 12.2 / 10.8 us, policy 24.8 / 24.3 / 22.6 us; 32768 tokens, policy 3.8 /
// 4.5 / 6.1 us).
struct PrefGrad {
  SeqArgs q;
  const float* coef;
  const float* grad_pair;
  float* grad_loss;
  struct Raw {
    int64_t target;
  };
  __device__ __forceinline__ void load(Raw& r, int t) const { r.target = q.targets[t]; }
  struct Seq {
    float grad;
  };
  __device__ __forceinline__ Seq open(int s) const { return {grad_pair[s >> 1] * coef[s]}; }
  __device__ __forceinline__ float grad(const Raw&, const Seq& s) const { return s.grad; }
};
struct PolicyGrad {
  PolicyArgs a;
  SeqArgs q;
  float* grad_loss;
  using Raw = PolicyRaw;
  __device__ __forceinline__ void load(Raw& r, int t) const { load_token(a, r, t); }
  struct Seq {
    float adv;
    double weight;
  };
  __device__ __forceinline__ Seq open(int s) const {
    return {a.per_token ? 0.f : a.adv[s],
            (double)a.grad_seq[s] * (q.mean ? 1.0 / (double)max(a.tokens[s], 1) : 1.0)};
  }
  __device__ __forceinline__ float grad(const Raw& r, const Seq& s) const {
    return (float)(s.weight * policy_token(a, r, (double)(a.per_token ? r.adv : s.adv)).slope);
  }
};
template <int J, class Op>
__global__ void __launch_bounds__(256) grad_kernel(Op op) {
  const SeqArgs& q = op.q;
  const int lane = lane_id();
  const int base = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 * J);
  if (base >= q.T) return;
  typename Op::Raw raw[J];
#pragma unroll
  for (int j = 0; j < J; ++j) op.load(raw[j], min(base + 64 * j + lane, q.T - 1));
  Window w;
  int s = w.open(q, base), end = w.end(q, s);
  if (q.S == 0) {
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (base + 64 * j + lane < q.T) op.grad_loss[base + 64 * j + lane] = 0.f;
    return;
  }
  typename Op::Seq here = op.open(clip(s, q));
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int b = base + 64 * j, e = min(b + 64, q.T);
    if (b >= q.T) break;
    int mine = s;
    typename Op::Seq seq = here;
    if (e > end) {
      mine = w.walk(q, b, e - 1);
      seq = op.open(clip(mine, q));
      s = __builtin_amdgcn_readlane(mine, 63);
      end = w.end(q, s);
      if (j + 1 < J) here = op.open(clip(s, q));
    }
    if (b + lane < e) {
      const bool counts = mine >= 0 && mine < q.S && raw[j].target != q.ignore_index;
      op.grad_loss[b + lane] = counts ? op.grad(raw[j], seq) : 0.f;
    }
  }
}

bool launched_ok() { return hipGetLastError() == hipSuccess; }

template <class Op, class Args, int LANES>
void launch_finish(const Args& a, int units, hipStream_t s) {
  constexpr int PER = 256 / LANES;
  hipLaunchKernelGGL((finish_kernel<Op, Args, LANES>), dim3((unsigned)(units + PER - 1) / PER), dim3(256), 0, s, a);
}

template <class Op, class Args>
bool forward(const Args& a, hipStream_t s) {
  const SeqArgs& q = a.q;
  if (q.S == 0) return true;
  const SeqPlan p = seq_plan(q.T, q.S);
  const int units = q.S / Op::PER_UNIT;
  if (p.chunks <= 16 && units <= 2048) {  // (a thread takes a few units at most)
    hipLaunchKernelGGL((small_kernel<Op, Args>), dim3(1), dim3(1024), 0, s, a);
    return launched_ok();
  }
  if (p.chunks > 0) {  // (no tokens: sequences without a part)
    const dim3 grid((unsigned)(p.chunks + 3) / 4);
    hipLaunchKernelGGL((chunk_kernel<Op, Args>), grid, dim3(256), 0, s, a);
    if (!launched_ok()) return false;
  }
  // a unit's parts side by side: a workgroup where there are many (one pair of 131071 tokens:
  // 4.5 us instead of 5.9 in a wavefront), eight lanes where there are more units than
  // wavefronts
  if (p.chunks >= 512 * (int64_t)units)
    launch_finish<Op, Args, 256>(a, units, s);
  else if (units <= 16384)
    launch_finish<Op, Args, 64>(a, units, s);
  else
    launch_finish<Op, Args, 8>(a, units, s);
  return launched_ok();
}
template <int J, class Op>
void launch_grad(const Op& op, hipStream_t s) {
  constexpr int PER = 256 * J;
  hipLaunchKernelGGL((grad_kernel<J, Op>), dim3((unsigned)(op.q.T + PER - 1) / PER), dim3(256), 0, s, op);
}

template <class Op>
bool backward(const Op& op, hipStream_t s) {
  const int T = op.q.T;
  if (T == 0) return true;
  if (T <= 64 * kWaves)
    launch_grad<1>(op, s);
  else
    launch_grad<4>(op, s);
  return launched_ok();
}

}  // namespace

SeqPlan seq_plan(int T, int S) {
  SeqPlan p;
  // Up to 2048 tokens the sixteen wavefronts of one workgroup, which then joins the sums in
  // the same launch (policy forward, us a call / replayed in a graph: T = 2000, 16 sequences
  // 8.3 / 6.4 instead of 11.5 / 5.7; T = 4000 8.8 / 8.7 instead of 11.5 / 5.7).
  const int most = T <= 2048 ? 16 : kWaves;
  p.chunk = 64 * std::max(1, (T + 64 * most - 1) / (64 * most));
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
