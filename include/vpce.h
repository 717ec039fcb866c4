/*
 * vpce.h: fused vocabulary-projection softmax cross-entropy for one GPU's share
 * of a Ring-DTP vocabulary projection (arXiv 2609.14306, Sec. 3.2 and the
 * appendix section on Ring-DTP, Algorithm 2), for AMD Instinct MI355X (gfx950).
 *
 * Problem (Sec. 3.2 notation in brackets):
 *   H        [T, d]   hidden states of the T local tokens          [X_r, N x H]
 *   W_p      [V_p, d] vocabulary shard p, row layout (one row per vocabulary
 *                     id), owning global ids [off_p, off_p + V_p) with
 *                     off_p = V_0 + ... + V_{p-1}                  [W_r^T, V_r]
 *   targets  [T]      int64 target ids, or ignore_index
 *   y_tv = h_t . w_v  logit of token t and vocabulary id v
 *
 * The forward visits the shards in `order` (the ring's visiting order: on rank
 * r of a move-weights ring that is r, r-1, ..., r-P+1 mod P, Algorithm 2) and
 * folds each block of logits into a running per-token state (m, s, y_target)
 * with the online-softmax update of Sec. 3.2; no logits tensor larger than a
 * fixed register tile is ever formed.  The backward recomputes each block of
 * logits from the saved normaliser lse, forms the softmax residual and
 * contracts it into the input and weight gradients (appendix on Ring-DTP),
 * staging the residual through a fixed-size strip buffer.  Every buffer the
 * library uses is allocated by the caller; the workspace size depends on T and
 * the strip budget, never on V.
 *
 * Conventions for every entry point:
 *   - device pointers are HIP device (or managed) memory on the current device;
 *     "host" arrays are ordinary CPU memory read before the call returns;
 *   - dense arrays are row-major and contiguous; H, every W_p and the workspace
 *     must be 16-byte aligned;
 *   - `stream` is a hipStream_t (NULL = the null stream); all work is enqueued
 *     on it and the call returns without synchronising (except vp_ce_check);
 *   - argument, shape, alignment and workspace errors are returned before any
 *     work is enqueued; a failed launch returns VP_ERR_HIP;
 *   - the library keeps no pointer after a call returns and has no global
 *     mutable state: calls on different streams with different workspaces may
 *     run concurrently.
 */
#ifndef VPCE_H
#define VPCE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define VPCE_ABI_VERSION 1
#define VP_MAX_SHARDS 64

typedef enum {
  VP_OK = 0,
  VP_ERR_NULL = 1,        /* a required pointer is NULL */
  VP_ERR_SHAPE = 2,       /* T out of [0, 2^23 - 256], d out of [8, 2^22] or d % 8 != 0,
                             P out of [1, VP_MAX_SHARDS], V_p out of [0, 2^30], sum V_p out of
                             [1, 2^31 - 1], strip_elems out of [0, 2^30] */
  VP_ERR_DTYPE = 3,       /* dtype is not VP_F32 / VP_BF16 */
  VP_ERR_ORDER = 4,       /* order is not a permutation of 0..P-1 */
  VP_ERR_ALIGN = 5,       /* a device pointer is not 16-byte aligned (4 for a fold state) */
  VP_ERR_WORKSPACE = 6,   /* workspace pointer NULL or smaller than the size the library asked for */
  VP_ERR_TARGET = 7,      /* (vp_ce_check) some target was outside [0, V) and not ignore_index */
  VP_ERR_HIP = 8,         /* a HIP runtime call or a kernel launch failed */
  VP_ERR_UNSUPPORTED = 9, /* valid request the library does not implement */
  VP_ERR_VALUE = 10       /* a parameter (eps, beta, a clip bound, ...) is outside its range */
} vp_status;

typedef enum {
  VP_F32 = 0,  /* H and W in float32; logits, residual and gradients in float32 */
  VP_BF16 = 1  /* H and W in bfloat16; products accumulated in float32; the residual
                  staged as bfloat16 (round to nearest even); gradients in float32 */
} vp_dtype;

/* flags */
#define VP_ACCUMULATE_DW 1u /* backward adds into dW_p instead of overwriting it: on a
                               move-weights ring the weight gradient travels with the
                               weight shard and collects every rank's contribution */

typedef struct {
  int64_t T;                  /* local tokens, 0..2^23 - 256 (T == 0 is a no-op) */
  int64_t d;                  /* hidden width, 8..2^22 and a multiple of 8 */
  int32_t P;                  /* number of vocabulary shards, 1..VP_MAX_SHARDS */
  int32_t dtype;              /* vp_dtype of H and W */
  const int64_t* shard_rows;  /* host [P]: V_p >= 0 rows of shard p, sum >= 1 */
  const int32_t* order;       /* host [P]: visiting order, a permutation of 0..P-1; NULL = 0..P-1 */
  int64_t ignore_index;       /* target value that marks a token without loss (e.g. -100) */
  uint32_t flags;             /* VP_ACCUMULATE_DW */
  int64_t strip_elems;        /* backward residual-strip budget in elements per layout,
                                 0..2^30; 0 = default (100 Mi) */
} vp_problem;

/* Workspace sizes in bytes for vp_ce_forward (*fwd_bytes) and vp_ce_backward
 * (*bwd_bytes); either output pointer may be NULL.  Host only, needs no device.
 * forward: per-token partial states of the vocabulary splits, O(T) (up to 2048
 * tokens the call may use more of them than it needs: a workspace with room for
 * 32 splits, 8 bytes x 32 x T beside the header and T floats, is accepted too);
 * backward: the residual strip in two layouts, twice (one being written while
 * the other is contracted: 4 x strip_elems elements at most), and room for H^T
 * (T x d elements, T rounded up to 256) and W^T of one vocabulary chunk (d x
 * strip columns), which hold transposed copies, longer strips or partial sums of
 * dH, whichever the call's plan takes.  Neither depends on V. */
vp_status vp_ce_workspace_size(const vp_problem* prob, size_t* fwd_bytes, size_t* bwd_bytes);

/* Forward (Sec. 3.2, Eq. of the online-softmax fold; Algorithm 2):
 *   lse[t]  = log sum_{v < V} exp(y_tv)                       (float32, device [T])
 *   loss[t] = lse[t] - y_{t, targets[t]},  0 if targets[t] == ignore_index,
 *             NaN if targets[t] is outside [0, V) (also counted for vp_ce_check)
 * H: device [T, d] of dtype; W_shards: host array of P device pointers, shard p
 * is [V_p, d] of dtype (NULL allowed when V_p == 0); targets: device int64 [T];
 * ws: device workspace of at least the forward size.  lse is the saved
 * normaliser the backward replays from. */
vp_status vp_ce_forward(const vp_problem* prob, const void* H, const void* const* W_shards,
                        const int64_t* targets, float* loss, float* lse, void* ws,
                        size_t ws_bytes, void* stream);

/* The forward for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): the same as
 * vp_ce_forward, with the same kernels and results, but its workspace is a
 * library-owned device buffer of 16 MiB per device (held from the first call on a
 * device until the process ends), so the call allocates nothing.  The caller still
 * passes H, the shards, the targets and the outputs.
 *   - Returns VP_ERR_WORKSPACE before any work is enqueued if the problem's forward
 *     workspace (vp_ce_workspace_size) exceeds 16 MiB (about T <= 460000 tokens at the
 *     usual split counts).
 *   - Every call on one device shares that device's buffer: calls that overlap on a
 *     device (different streams or threads) race and give wrong results; calls
 *     ordered on one stream are safe.
 *   - The count of out-of-range targets is kept in that buffer and is not reported
 *     (vp_ce_check needs a caller's workspace); such tokens still get a NaN loss.
 *   - The first call on a device looks up the buffer's device address (no
 *     allocation); VP_ERR_HIP if that fails. */
vp_status vp_ce_forward_noalloc(const vp_problem* prob, const void* H,
                                const void* const* W_shards, const int64_t* targets,
                                float* loss, float* lse, void* stream);

/* Backward (appendix on Ring-DTP: recompute each block of logits from the saved
 * normaliser, form the softmax residual, contract into both gradients):
 *   G[t, v]  = grad_loss[t] * (exp(y_tv - lse[t]) - [v == targets[t]]),
 *              0 on ignored tokens, NaN on out-of-range targets
 *   dH       = G W            device float32 [T, d], overwritten
 *   dW_p     = G[:, shard p]^T H   device float32 [V_p, d] per shard (host array of
 *              P device pointers; NULL allowed when V_p == 0), overwritten, or
 *              added to with VP_ACCUMULATE_DW
 * lse: device float32 [T] from vp_ce_forward on the same inputs; grad_loss:
 * device float32 [T] upstream gradient of each token's loss (1/N_valid for a
 * mean, 1 for a sum). */
vp_status vp_ce_backward(const vp_problem* prob, const void* H, const void* const* W_shards,
                         const int64_t* targets, const float* lse, const float* grad_loss,
                         float* dH, float* const* dW_shards, void* ws, size_t ws_bytes,
                         void* stream);

/* Per-shard fold: one meeting of Algorithm 2 at a time, for a per-token state
 * that travels with the activations (move-activations: the hidden states, the
 * targets and the state visit the ranks that hold the vocabulary shards, and a
 * final hop returns the state to its owner, Sec. 3.2 and Algorithm 2).
 *
 * State: device float32 [3 * T], three planes of T values:
 *   m[t]  = state[t]          running maximum logit over the vocabulary ids folded so
 *                             far (natural units), -inf before the first shard;
 *   s[t]  = state[T + t]      sum over those ids of exp(y_tv - m[t]);
 *   y[t]  = state[2T + t]     the target logit h_t . w_{targets[t]} once the shard
 *                             owning targets[t] has been folded, 0 before.
 * The planes are plain numbers in host byte order: the state is serialised by
 * copying its 12 T bytes, on any device or the host, and folding may resume
 * from such a copy on another device.  Folding is order-free up to rounding
 * (the online-softmax update is associative and commutative). */

/* state <- (-inf, 0, 0) for every token.  state: device float32 [3 * T], 4-byte
 * aligned; T in [0, 2^23 - 256] (VP_ERR_SHAPE otherwise). */
vp_status vp_ce_state_init(float* state, int64_t T, void* stream);

/* Folds one vocabulary shard into the state (the online-softmax update of Sec. 3.2):
 *   m' = max(m, max_v y_tv),  s' = s e^(m - m') + sum_v e^(y_tv - m'),
 *   y' = y_{t, targets[t]} where id_offset <= targets[t] < id_offset + V_q, else y.
 * shard: a vp_problem with P == 1 whose shard_rows[0] = V_q are the shard's rows
 * (T, d, dtype as for vp_ce_forward; order NULL or {0}; ignore_index, flags and
 * strip_elems unused); id_offset: the global vocabulary id of the shard's first
 * row (id_offset + V_q <= 2^31 - 1).  H: device [T, d]; W_shard: device [V_q, d]
 * (NULL allowed when V_q == 0); targets: device int64 [T] of global ids; state as
 * above, updated in place.  ws: the forward workspace of `shard`
 * (vp_ce_workspace_size(shard, &fwd, NULL); it depends on T, d and dtype, never on
 * V_q), 16-byte aligned.  V_q == 0 or T == 0 returns VP_OK before anything else is
 * checked or launched and leaves the state unchanged: ws, H, W_shard, targets and
 * state may then be NULL. */
vp_status vp_ce_fold_shard(const vp_problem* shard, int64_t id_offset, const void* H,
                           const void* W_shard, const int64_t* targets, float* state, void* ws,
                           size_t ws_bytes, void* stream);

/* From a state that has met every shard of the vocabulary described by `prob`
 * (V = sum of its shard_rows; T and ignore_index as for vp_ce_forward):
 *   lse[t]  = m[t] + log s[t],
 *   loss[t] = lse[t] - y[t], 0 if targets[t] == ignore_index, NaN if targets[t] is
 *             outside [0, V) (counted in ws for vp_ce_check).
 * The state is only read.  ws: at least 256 bytes (the forward workspace of any
 * problem is enough), 16-byte aligned. */
vp_status vp_ce_fold_finalize(const vp_problem* prob, const int64_t* targets, const float* state,
                              float* loss, float* lse, void* ws, size_t ws_bytes, void* stream);

/* How vp_ce_backward cuts a problem (host only, needs no device): the residual
 * strip is Tc tokens by at most Vc vocabulary rows; `strips` strips cover the
 * T x V residual (a shard of more than Vc rows cut into balanced vocabulary
 * chunks, smaller consecutive shards of at least 256 rows sharing a strip while
 * they fit, each meeting every token chunk), and the backward makes
 * stage_launches = strips + 1 launches of its fused recompute / residual / dH / dW
 * kernel (0 when T == 0). */
typedef struct {
  int64_t Tc;
  int64_t Vc;
  int64_t strips;
  int64_t stage_launches;
} vp_plan_info;
vp_status vp_ce_plan_info(const vp_problem* prob, vp_plan_info* info);

/* Reads the count of out-of-range targets that the last forward or backward on
 * this workspace found (synchronises `stream`).  Returns VP_ERR_TARGET if it is
 * non-zero.  *bad_targets may be NULL. */
vp_status vp_ce_check(const void* ws, void* stream, int64_t* bad_targets);

/* ------------------------------------------------------------------------------
 * Layer norm of the hidden states, in front of the projection (H of vp_ce_forward is
 * its Y; its dY is the dH of vp_ce_backward):
 *   mu_t  = (1/d) sum_j x_tj                        (0 with VP_NORM_RMS)
 *   r_t   = ((1/d) sum_j (x_tj - mu_t)^2 + eps)^(-1/2)
 *   y_tj  = gamma_j (x_tj - mu_t) r_t + beta_j
 * Sums are float32 (the sum of a row's squares among them: where it leaves float32, as with one
 * element of 2e19, rstd is 0); y is rounded once, to nearest even. */
#define VP_NORM_RMS 2u /* no mean: mu_t = 0 in the forward and the backward */

typedef struct {
  int64_t T;      /* tokens, 0..2^23 - 256 (T == 0: nothing to do in the forward) */
  int64_t d;      /* width, 8..16384 and a multiple of 8 (VP_ERR_SHAPE otherwise) */
  int32_t dtype;  /* vp_dtype of X, gamma, beta and Y */
  uint32_t flags; /* VP_NORM_RMS, VP_ACCUMULATE_DW */
  double eps;     /* 0, or within float32's normal numbers, 1.2e-38..3.4e38 (VP_ERR_VALUE otherwise) */
} vp_norm;

/* Workspace of vp_norm_backward in bytes.  Host only. */
vp_status vp_norm_workspace_size(const vp_norm* norm, size_t* bwd_bytes);

/* X: device [T, d] of dtype; gamma, beta: device [d] of dtype, beta may be NULL (no
 * bias); Y: device [T, d] of dtype, no part of X; mean, rstd: device float32 [T], what
 * the backward replays from (mean is neither written nor read with VP_NORM_RMS and may
 * then be NULL).  X, gamma, beta and Y must be 16-byte aligned. */
vp_status vp_norm_forward(const vp_norm* norm, const void* X, const void* gamma, const void* beta,
                          void* Y, float* mean, float* rstd, void* stream);

/* With xh_tj = (x_tj - mu_t) r_t and g_tj = dy_tj gamma_j:
 *   dx_tj    = r_t (g_tj - (1/d) sum_k g_tk - xh_tj (1/d) sum_k g_tk xh_tk)
 *              (without the first sum with VP_NORM_RMS)
 *   dgamma_j = sum_t dy_tj xh_tj,   dbeta_j = sum_t dy_tj
 * dY: device float32 [T, d]; dX: device float32 [T, d], overwritten; it may be dY
 * itself.  dgamma, dbeta: device float32 [d], overwritten, or added to with
 * VP_ACCUMULATE_DW; dbeta may be NULL (not computed).  All but mean and rstd must be
 * 16-byte aligned, and so must ws.  T == 0 gives dgamma = dbeta = 0 (or leaves them
 * when accumulating).  Two calls on the same inputs give the same bits. */
vp_status vp_norm_backward(const vp_norm* norm, const void* X, const void* gamma, const float* mean,
                           const float* rstd, const float* dY, float* dX, float* dgamma,
                           float* dbeta, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------------
 * Losses of whole sequences, behind the projection.  They read the per-token loss of
 * vp_ce_forward (loss_t = -log p of the target) and write the per-token gradient that
 * vp_ce_backward takes as grad_loss.
 *
 * The T tokens hold S sequences one after the other: sequence s is the tokens
 * start[s] .. start[s + 1] - 1 (start: device int32 [S + 1], never decreasing, within
 * 0..T; a sequence may be empty; tokens before start[0] or from start[S] on belong to
 * none).  A token counts if it belongs to a sequence and targets[t] != ignore_index:
 * what any other token's entry of a per-token array holds is not used (it may be NaN),
 * and its gradient is 0.  A counting token whose loss is NaN (an out-of-range target)
 * makes the results of its sequence, or of its pair, NaN, and no others.
 * With n_s the counting tokens of sequence s, a sum over it is weighted by c_s = 1, or
 * with VP_SEQ_MEAN by c_s = 1 / n_s (0 where n_s == 0).  Sums are float64, results are
 * rounded once to float32.
 *
 * Every offset is held against 0..T before it is used as one: wrong offsets never lead
 * outside an array.  A sequence whose own two offsets decrease or leave 0..T gets NaN
 * results; what the other sequences of such a call get is not specified. */
#define VP_SEQ_MEAN 4u

typedef struct {
  int64_t T;            /* tokens, 0..2^23 - 256 */
  int64_t S;            /* sequences, 0..2^22 */
  int64_t ignore_index; /* target value of a token that does not count */
  uint32_t flags;       /* VP_SEQ_MEAN */
} vp_sequences;

/* Workspace of vp_pref_forward and of vp_policy_forward in bytes.  Host only. */
vp_status vp_seq_workspace_size(const vp_sequences* seq, size_t* bytes);

typedef enum {
  VP_PREF_LOGISTIC = 0,
  VP_PREF_SQUARED = 1
} vp_pref_kind;

/* Preference loss over pairs: pair i is sequence 2i (preferred) and 2i + 1 (rejected),
 * so S must be even (VP_ERR_SHAPE otherwise).  With R_s = c_s sum_t (ref_t - loss_t),
 * the log ratio of the policy to the reference:
 *   reward_s = beta R_s,   z_i = reward_2i - reward_{2i+1} - margin
 *   VP_PREF_LOGISTIC: pair_loss_i = (1 - smoothing) log(1 + e^-z) + smoothing log(1 + e^z)
 *   VP_PREF_SQUARED:  pair_loss_i = ((z - 1/2) / beta)^2 */
typedef struct {
  int32_t kind;     /* vp_pref_kind (VP_ERR_VALUE otherwise, as for the rest) */
  double beta;      /* > 0 and finite */
  double margin;    /* finite */
  double smoothing; /* 0..1/2, 0 for VP_PREF_SQUARED */
} vp_preference;

/* targets: device int64 [T]; loss, ref_loss: device float32 [T], ref_loss may be NULL
 * (ref_t = 0); pair_loss: device float32 [S/2]; reward: device float32 [S];
 * coef: device float32 [S], what the backward replays from: d pair_loss / d loss_t for
 * the counting tokens of each sequence.  ws: 16-byte aligned. */
vp_status vp_pref_forward(const vp_sequences* seq, const vp_preference* pref, const int32_t* start,
                          const int64_t* targets, const float* loss, const float* ref_loss,
                          float* pair_loss, float* reward, float* coef, void* ws, size_t ws_bytes,
                          void* stream);

/* grad_loss[t] = grad_pair[s/2] coef[s] for the counting tokens of sequence s, else 0;
 * device float32 [T], every entry written.  grad_pair: device float32 [S/2], the
 * upstream gradient of each pair's loss.  start and targets as in the forward. */
vp_status vp_pref_backward(const vp_sequences* seq, const int32_t* start, const int64_t* targets,
                           const float* coef, const float* grad_pair, float* grad_loss,
                           void* stream);

/* Clipped policy loss with a KL term.  With A the advantage, rho_t = e^(old_t - loss_t)
 * and q_t = loss_t - ref_t:
 *   kl_t = e^q - q - 1          (estimates KL(policy || reference); >= 0)
 *   l_t  = -min(rho_t A, clip(rho_t, 1 - clip_low, 1 + clip_high) A) + kl_coef kl_t
 *   seq_loss_s = c_s sum_t l_t,   seq_kl_s = c_s sum_t kl_t
 * A token is clipped where the minimum is the clipped term alone (A > 0 and rho_t >
 * 1 + clip_high, or A < 0 and rho_t < 1 - clip_low; decided in float64): there the
 * first term has no gradient.  (A mean over all tokens of the batch is the form without
 * VP_SEQ_MEAN, with grad_seq = 1 / the sum of tokens.) */
#define VP_ADV_PER_TOKEN 8u

typedef struct {
  double clip_low;  /* 0..1 (VP_ERR_VALUE otherwise, as for the rest) */
  double clip_high; /* >= 0, may be infinite */
  double kl_coef;   /* >= 0 and finite */
  uint32_t flags;   /* VP_ADV_PER_TOKEN */
} vp_policy;

/* loss, old_loss, ref_loss: device float32 [T]; old_loss may be NULL (the policy that
 * drew the tokens is this one: rho = 1 with the gradient of rho), ref_loss may be NULL
 * (kl_t = 0); advantage: device float32 [S], or [T] with VP_ADV_PER_TOKEN; seq_loss,
 * seq_kl: device float32 [S]; clipped, tokens: device int32 [S], the clipped and the
 * counting tokens.  ws: 16-byte aligned. */
vp_status vp_policy_forward(const vp_sequences* seq, const vp_policy* policy, const int32_t* start,
                            const int64_t* targets, const float* loss, const float* old_loss,
                            const float* ref_loss, const float* advantage, float* seq_loss,
                            float* seq_kl, int32_t* clipped, int32_t* tokens, void* ws,
                            size_t ws_bytes, void* stream);

/* grad_loss[t] = grad_seq[s] c_s (A rho_t [not clipped] + kl_coef (e^q - 1)) for the
 * counting tokens of sequence s, else 0; device float32 [T], every entry written.
 * grad_seq: device float32 [S], the upstream gradient of each seq_loss; tokens: from
 * the forward (read with VP_SEQ_MEAN alone); the rest as in the forward. */
vp_status vp_policy_backward(const vp_sequences* seq, const vp_policy* policy, const int32_t* start,
                             const int64_t* targets, const float* loss, const float* old_loss,
                             const float* ref_loss, const float* advantage, const int32_t* tokens,
                             const float* grad_seq, float* grad_loss, void* stream);

const char* vp_status_str(vp_status s);
int vp_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* VPCE_H */
