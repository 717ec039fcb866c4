// Host side of the operators around the projection (layer norm, preference loss,
// policy loss) declared in include/vpce.h: argument checks and launches.  Every refusal
// is made before any HIP call, so these paths run on a machine without a GPU.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cfloat>
#include <cmath>

#include "vpce_head.h"

namespace {

constexpr int64_t kMaxT = (1ll << 23) - 256;  // as for vp_problem
constexpr int64_t kMaxNormD = 16384;          // a row stays in the registers of one workgroup
constexpr int64_t kMaxS = 1ll << 22;

inline bool off(const void* p, uintptr_t align) { return ((uintptr_t)p & (align - 1)) != 0; }

vp_status validate(const vp_norm* n) {
  if (!n) return VP_ERR_NULL;
  if (n->dtype != VP_F32 && n->dtype != VP_BF16) return VP_ERR_DTYPE;
  if (n->T < 0 || n->T > kMaxT || n->d < 8 || n->d % 8 != 0 || n->d > kMaxNormD) return VP_ERR_SHAPE;
  if (!(n->eps >= 0.0) || !std::isfinite(n->eps)) return VP_ERR_VALUE;
  // (the kernels hold it in float32: no other value may become 0 or infinite there)
  if (n->eps != 0.0 && (n->eps < FLT_MIN || n->eps > FLT_MAX)) return VP_ERR_VALUE;
  return VP_OK;
}

// One row of d sums for each partial dgamma and dbeta.
size_t norm_ws_bytes(const vp_norm* n) {
  return 256 + 2 * (size_t)vpce::norm_parts(n->T, (int)n->d) * (size_t)n->d * 4;
}

vp_status validate(const vp_sequences* q) {
  if (!q) return VP_ERR_NULL;
  if (q->T < 0 || q->T > kMaxT || q->S < 0 || q->S > kMaxS) return VP_ERR_SHAPE;
  return VP_OK;
}

size_t seq_ws_bytes(const vp_sequences* q) {
  return 256 + (size_t)vpce::seq_plan((int)q->T, (int)q->S).slots * vpce::kMaxSeqSums * sizeof(double);
}

vp_status validate(const vp_preference* p) {
  if (!p) return VP_ERR_NULL;
  if (p->kind != VP_PREF_LOGISTIC && p->kind != VP_PREF_SQUARED) return VP_ERR_VALUE;
  if (!(p->beta > 0.0) || !std::isfinite(p->beta) || !std::isfinite(p->margin)) return VP_ERR_VALUE;
  if (!(p->smoothing >= 0.0 && p->smoothing <= 0.5)) return VP_ERR_VALUE;
  if (p->kind == VP_PREF_SQUARED && p->smoothing != 0.0) return VP_ERR_VALUE;
  return VP_OK;
}

vp_status validate(const vp_policy* p) {
  if (!p) return VP_ERR_NULL;
  if (!(p->clip_low >= 0.0 && p->clip_low <= 1.0) || !(p->clip_high >= 0.0)) return VP_ERR_VALUE;
  if (!(p->kl_coef >= 0.0) || !std::isfinite(p->kl_coef)) return VP_ERR_VALUE;
  return VP_OK;
}

vp_status check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return VP_ERR_WORKSPACE;
  return off(ws, 16) ? VP_ERR_ALIGN : VP_OK;
}

// Offsets and targets of a call that has them.
vp_status check_tokens(const vp_sequences* q, const int32_t* start, const int64_t* targets) {
  if (q->S > 0 && !start) return VP_ERR_NULL;
  if (q->T > 0 && !targets) return VP_ERR_NULL;
  return off(start, 4) || off(targets, 8) ? VP_ERR_ALIGN : VP_OK;
}

vpce::SeqArgs seq_args(const vp_sequences* q, const int32_t* start, const int64_t* targets,
                       void* ws = nullptr) {
  vpce::SeqArgs a;
  a.start = start;
  a.targets = targets;
  a.ignore_index = q->ignore_index;
  a.T = (int32_t)q->T;
  a.S = (int32_t)q->S;
  a.mean = (q->flags & VP_SEQ_MEAN) != 0;
  a.chunk = vpce::seq_plan(a.T, a.S).chunk;
  a.part = (double*)ws;
  return a;
}

vp_status policy_args(const vp_sequences* seq, const vp_policy* p, const int32_t* start,
                      const int64_t* targets, const float* loss, const float* old_loss,
                      const float* ref_loss, const float* advantage, vpce::PolicyArgs* a) {
  vp_status st = validate(seq);
  if (st != VP_OK) return st;
  if ((st = validate(p)) != VP_OK) return st;
  if ((st = check_tokens(seq, start, targets)) != VP_OK) return st;
  const bool per_token = (p->flags & VP_ADV_PER_TOKEN) != 0;
  if (seq->T > 0 && !loss) return VP_ERR_NULL;
  if ((per_token ? seq->T : seq->S) > 0 && !advantage) return VP_ERR_NULL;
  if (off(loss, 4) || off(old_loss, 4) || off(ref_loss, 4) || off(advantage, 4)) return VP_ERR_ALIGN;
  *a = vpce::PolicyArgs{};
  a->q = seq_args(seq, start, targets);
  a->loss = loss;
  a->old = old_loss ? old_loss : loss;
  a->ref = ref_loss ? ref_loss : loss;
  a->adv = advantage;
  a->adv_tok = per_token ? advantage : loss;
  a->has_old = old_loss != nullptr;
  a->has_ref = ref_loss != nullptr;
  a->per_token = per_token;
  a->low = 1.0 - p->clip_low;
  a->high = 1.0 + p->clip_high;
  a->log_low = std::log1p(-p->clip_low);
  a->log_high = std::log1p(p->clip_high);
  a->kl_coef = p->kl_coef;
  return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_norm_workspace_size(const vp_norm* norm, size_t* bwd_bytes) {
  const vp_status st = validate(norm);
  if (st != VP_OK) return st;
  if (bwd_bytes) *bwd_bytes = norm_ws_bytes(norm);
  return VP_OK;
}

vp_status vp_norm_forward(const vp_norm* norm, const void* X, const void* gamma, const void* beta,
                          void* Y, float* mean, float* rstd, void* stream) {
  const vp_status st = validate(norm);
  if (st != VP_OK) return st;
  const bool rms = (norm->flags & VP_NORM_RMS) != 0;
  if (norm->T == 0) return VP_OK;
  if (!X || !gamma || !Y || !rstd || (!rms && !mean)) return VP_ERR_NULL;
  if (off(X, 16) || off(gamma, 16) || off(beta, 16) || off(Y, 16)) return VP_ERR_ALIGN;
  if (off(rstd, 4) || (!rms && off(mean, 4))) return VP_ERR_ALIGN;
  vpce::NormArgs a;
  a.X = X;
  a.gamma = gamma;
  a.beta = beta;
  a.Y = Y;
  a.mean = rms ? nullptr : mean;
  a.rstd = rstd;
  a.T = norm->T;
  a.d = (int32_t)norm->d;
  a.eps = (float)norm->eps;
  return vpce::run_norm_forward(norm->dtype, rms, a, (hipStream_t)stream) ? VP_OK : VP_ERR_HIP;
}

vp_status vp_norm_backward(const vp_norm* norm, const void* X, const void* gamma, const float* mean,
                           const float* rstd, const float* dY, float* dX, float* dgamma,
                           float* dbeta, void* ws, size_t ws_bytes, void* stream) {
  vp_status st = validate(norm);
  if (st != VP_OK) return st;
  const bool rms = (norm->flags & VP_NORM_RMS) != 0;
  if ((st = check_ws(ws, ws_bytes, norm_ws_bytes(norm))) != VP_OK) return st;
  if (!gamma || !dgamma) return VP_ERR_NULL;
  if (norm->T > 0 && (!X || !rstd || !dY || !dX || (!rms && !mean))) return VP_ERR_NULL;
  if (off(X, 16) || off(gamma, 16) || off(dY, 16) || off(dX, 16) || off(dgamma, 16) || off(dbeta, 16))
    return VP_ERR_ALIGN;
  if (off(rstd, 4) || (!rms && off(mean, 4))) return VP_ERR_ALIGN;
  vpce::NormGradArgs a;
  a.X = X;
  a.gamma = gamma;
  a.mean = rms ? nullptr : mean;
  a.rstd = rstd;
  a.dY = dY;
  a.dX = dX;
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.part = (float*)ws;
  a.T = norm->T;
  a.d = (int32_t)norm->d;
  a.accumulate = (norm->flags & VP_ACCUMULATE_DW) != 0;
  return vpce::run_norm_backward(norm->dtype, rms, a, (hipStream_t)stream) ? VP_OK : VP_ERR_HIP;
}

vp_status vp_seq_workspace_size(const vp_sequences* seq, size_t* bytes) {
  const vp_status st = validate(seq);
  if (st != VP_OK) return st;
  if (bytes) *bytes = seq_ws_bytes(seq);
  return VP_OK;
}

vp_status vp_pref_forward(const vp_sequences* seq, const vp_preference* pref, const int32_t* start,
                          const int64_t* targets, const float* loss, const float* ref_loss,
                          float* pair_loss, float* reward, float* coef, void* ws, size_t ws_bytes,
                          void* stream) {
  vp_status st = validate(seq);
  if (st != VP_OK) return st;
  if (seq->S % 2 != 0) return VP_ERR_SHAPE;
  if ((st = validate(pref)) != VP_OK) return st;
  if ((st = check_ws(ws, ws_bytes, seq_ws_bytes(seq))) != VP_OK) return st;
  if ((st = check_tokens(seq, start, targets)) != VP_OK) return st;
  if (seq->T > 0 && !loss) return VP_ERR_NULL;
  if (seq->S > 0 && (!pair_loss || !reward || !coef)) return VP_ERR_NULL;
  if (off(loss, 4) || off(ref_loss, 4) || off(pair_loss, 4) || off(reward, 4) || off(coef, 4))
    return VP_ERR_ALIGN;
  vpce::PrefArgs a;
  a.q = seq_args(seq, start, targets, ws);
  a.loss = loss;
  a.ref = ref_loss ? ref_loss : loss;
  a.has_ref = ref_loss != nullptr;
  a.kind = pref->kind;
  a.beta = pref->beta;
  a.margin = pref->margin;
  a.smoothing = pref->smoothing;
  a.pair_loss = pair_loss;
  a.reward = reward;
  a.coef = coef;
  return vpce::run_pref_forward(a, (hipStream_t)stream) ? VP_OK : VP_ERR_HIP;
}

vp_status vp_pref_backward(const vp_sequences* seq, const int32_t* start, const int64_t* targets,
                           const float* coef, const float* grad_pair, float* grad_loss,
                           void* stream) {
  vp_status st = validate(seq);
  if (st != VP_OK) return st;
  if (seq->S % 2 != 0) return VP_ERR_SHAPE;
  if ((st = check_tokens(seq, start, targets)) != VP_OK) return st;
  if (seq->S > 0 && (!coef || !grad_pair)) return VP_ERR_NULL;
  if (seq->T > 0 && !grad_loss) return VP_ERR_NULL;
  if (off(coef, 4) || off(grad_pair, 4) || off(grad_loss, 4)) return VP_ERR_ALIGN;
  return vpce::run_pref_backward(seq_args(seq, start, targets), coef, grad_pair, grad_loss, (hipStream_t)stream)
             ? VP_OK
             : VP_ERR_HIP;
}

vp_status vp_policy_forward(const vp_sequences* seq, const vp_policy* policy, const int32_t* start,
                            const int64_t* targets, const float* loss, const float* old_loss,
                            const float* ref_loss, const float* advantage, float* seq_loss,
                            float* seq_kl, int32_t* clipped, int32_t* tokens, void* ws,
                            size_t ws_bytes, void* stream) {
  vpce::PolicyArgs a;
  vp_status st = policy_args(seq, policy, start, targets, loss, old_loss, ref_loss, advantage, &a);
  if (st != VP_OK) return st;
  if ((st = check_ws(ws, ws_bytes, seq_ws_bytes(seq))) != VP_OK) return st;
  if (seq->S > 0 && (!seq_loss || !seq_kl || !clipped || !tokens)) return VP_ERR_NULL;
  if (off(seq_loss, 4) || off(seq_kl, 4) || off(clipped, 4) || off(tokens, 4)) return VP_ERR_ALIGN;
  a.q.part = (double*)ws;
  a.seq_loss = seq_loss;
  a.seq_kl = seq_kl;
  a.clipped = clipped;
  a.tokens = tokens;
  return vpce::run_policy_forward(a, (hipStream_t)stream) ? VP_OK : VP_ERR_HIP;
}

vp_status vp_policy_backward(const vp_sequences* seq, const vp_policy* policy, const int32_t* start,
                             const int64_t* targets, const float* loss, const float* old_loss,
                             const float* ref_loss, const float* advantage, const int32_t* tokens,
                             const float* grad_seq, float* grad_loss, void* stream) {
  vpce::PolicyArgs a;
  const vp_status st = policy_args(seq, policy, start, targets, loss, old_loss, ref_loss, advantage, &a);
  if (st != VP_OK) return st;
  if (seq->S > 0 && (!grad_seq || (a.q.mean && !tokens))) return VP_ERR_NULL;
  if (seq->T > 0 && !grad_loss) return VP_ERR_NULL;
  if (off(tokens, 4) || off(grad_seq, 4) || off(grad_loss, 4)) return VP_ERR_ALIGN;
  a.tokens = const_cast<int32_t*>(tokens);
  a.grad_seq = grad_seq;
  a.grad_loss = grad_loss;
  return vpce::run_policy_backward(a, (hipStream_t)stream) ? VP_OK : VP_ERR_HIP;
}

}  // extern "C"
