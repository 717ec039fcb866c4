// Internal interface between the host side of the operators around the projection
// (vpce_head_api.cpp) and their kernels (vpce_norm.hip, vpce_seq.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vpce.h"

namespace vpce {

struct NormArgs {
  const void* X;      // [T, d]
  const void* gamma;  // [d]
  const void* beta;   // [d] or null
  void* Y;            // [T, d]
  float* mean;        // [T], null without a mean
  float* rstd;        // [T]
  int64_t T;
  int32_t d;
  float eps;
};

struct NormGradArgs {
  const void* X;
  const void* gamma;
  const float* mean;  // null without a mean
  const float* rstd;
  const float* dY;  // [T, d]
  float* dX;        // [T, d], may be dY
  float* dgamma;    // [d]
  float* dbeta;     // [d] or null
  float* part;      // workspace: [2][norm_parts][d]
  int64_t T;
  int32_t d;
  int32_t accumulate;
};

// Rows of partial sums of dgamma (and of dbeta) that a backward writes.
int norm_parts(int64_t T, int d);
bool run_norm_forward(int dtype, bool rms, const NormArgs& a, hipStream_t s);
bool run_norm_backward(int dtype, bool rms, const NormGradArgs& a, hipStream_t s);

// T packed tokens in S sequences (start [S + 1]); see vpce.h.
struct SeqArgs {
  const int32_t* start;
  const int64_t* targets;
  int64_t ignore_index;
  int32_t T, S;
  int32_t mean;
  int32_t chunk;  // tokens of a chunk
  double* part;   // workspace: [slots][sums]; the forwards' alone
};

// How the tokens of a forward are cut, and its partial sums.
struct SeqPlan {
  int32_t chunk, chunks;
  int64_t slots;
};
SeqPlan seq_plan(int T, int S);
constexpr int kMaxSeqSums = 3;  // of one slot

// Arrays that a call leaves out are the loss in these, and what is read from them is not
// used: every token's loads go out together, without a branch between them.
struct PrefArgs {
  SeqArgs q;
  const float* loss;
  const float* ref;
  int32_t has_ref, kind;
  double beta, margin, smoothing;
  float *pair_loss, *reward, *coef;
};

struct PolicyArgs {
  SeqArgs q;
  const float* loss;
  const float *old, *ref;
  const float* adv;      // [S], or unused
  const float* adv_tok;  // [T], or unused
  int32_t has_old, has_ref, per_token;
  double low, high;          // clip bounds of the ratio
  double log_low, log_high;  // and their logarithms
  double kl_coef;
  float *seq_loss, *seq_kl;
  int32_t *clipped, *tokens;  // the backward reads tokens
  const float* grad_seq;
  float* grad_loss;
};

bool run_pref_forward(const PrefArgs& a, hipStream_t s);
bool run_pref_backward(const SeqArgs& q, const float* coef, const float* grad_pair, float* grad_loss,
                       hipStream_t s);
bool run_policy_forward(const PolicyArgs& a, hipStream_t s);
bool run_policy_backward(const PolicyArgs& a, hipStream_t s);

}  // namespace vpce
