// HIP kernels for gfx950 (MI355X): fused vocabulary-projection softmax
// cross-entropy, forward with an online log-sum-exp fold and backward with
// logits recompute (arXiv 2609.14306, Sec. 3.2 and the appendix on Ring-DTP).
//
// One MFMA GEMM mainloop, C[m][n] = sum_k A[m][k] B[n][k], serves the four
// contractions of the path:
//   logits (forward and recompute)  C[v][t] = sum_k W[v][k]   H[t][k]
//   dH                              C[t][n] = sum_v G^T[t][v] W[v][n]
//   dW                              C[v][n] = sum_t G[v][t]   H[t][n]
// The backward stores the softmax residual of a (vocabulary chunk, token chunk) strip
// in both layouts (G and G^T), k-contiguous for both contractions.  Their other operand,
// W or H, has its contraction index as its row index: it is read through gfx950's LDS
// transpose read (two 8-byte reads per fragment instead of one of 16, 1.5% of the
// mainloop's rate), or, where tokens are many enough to pay for them, from k-contiguous
// transposed copies (0.47 ms for V = 201088, d = 2880 whatever T is; plan_bwd).
//
// Logits are computed transposed (vocabulary rows, token columns) so that in the
// MFMA accumulator layout every lane owns whole token columns: the online
// softmax state of a token lives in one lane's registers and needs no
// cross-lane traffic until the very end of a workgroup's vocabulary range.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <mutex>

#include "vpce_backward.h"
#include "vpce_internal.h"
#include "vpce_tiles.h"

namespace vpce {

__global__ void ws_init_kernel(unsigned long long* counter) {
  if (threadIdx.x == 0 && blockIdx.x == 0) *counter = 0ull;
}

__global__ void fill_zero_kernel(float* p, int64_t n) {
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) p[i] = 0.f;
}

// End of a forward workgroup: merges the two lane halves that share a token column,
// then the wave rows, and writes the workgroup's partial state per token.  LDS must
// be idle; the header's counter is cleared for the merge kernel that follows.
template <class G>
__device__ __forceinline__ void write_partials(const FwdArgs& a, float (&m_run)[G::NB],
                                               float (&s_run)[G::NB], int split, int n0, float* red) {
  constexpr int BN = G::BN, NB = G::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = G::wave_n(wave);
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const float mo = __shfl_xor(m_run[j], 32);
    const float so = __shfl_xor(s_run[j], 32);
    merge_state(m_run[j], s_run[j], mo, so);
  }
  __syncthreads();
  const int wr = wave / G::WGN;  // red: [WGM][2][BN]
  if (lane < 32) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      red[(wr * 2) * BN + wn + 32 * j + lane] = m_run[j];
      red[(wr * 2 + 1) * BN + wn + 32 * j + lane] = s_run[j];
    }
  }
  __syncthreads();
  if (wr == 0 && lane < 32) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int c = wn + 32 * j + lane;
      for (int w2 = 1; w2 < G::WGM; ++w2)
        merge_state(m_run[j], s_run[j], red[(w2 * 2) * BN + c], red[(w2 * 2 + 1) * BN + c]);
      const int64_t n = n0 + c;
      if (n < a.T) {
        a.m_part[(int64_t)split * a.T + n] = m_run[j] == kNoLogit ? -INFINITY : m_run[j];
        a.s_part[(int64_t)split * a.T + n] = s_run[j];
      }
    }
  }
  if (blockIdx.x == 0 && tid == 0 && a.counter) *a.counter = 0ull;
}

// Forward: each workgroup owns BN tokens and one contiguous range of the
// vocabulary tiles in visiting order; it folds every logits tile into a
// per-lane online-softmax state, gathers the target logit from the one tile
// whose rows contain it, and writes its partial (m, s) per token.
template <class E, class G>
__global__ void __launch_bounds__(G::NT, G::OCC) fwd_kernel(FwdArgs a) {
  using S = typename E::storage;
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB;
  __shared__ __attribute__((aligned(16))) S smem[G::LDS_ELEMS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = G::wave_m(wave), wn = G::wave_n(wave);
  // split fastest: the workgroups an XCD runs together share token blocks (H panels)
  // across splits and vocabulary tiles (W panels) across token blocks.
  const int logical = xcd_logical(blockIdx.x, gridDim.x);
  const int tb = logical / a.n_splits;
  const int split = logical % a.n_splits;
  const int n0 = tb * BN;
  const int t_begin = (int)((int64_t)split * a.n_tiles / a.n_splits);
  const int t_end = (int)((int64_t)(split + 1) * a.n_tiles / a.n_splits);

  float m_run[NB], s_run[NB];
  int64_t tgt[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    m_run[j] = kNoLogit;
    s_run[j] = 0.f;
    const int64_t n = n0 + wn + 32 * j + (lane & 31);
    tgt[j] = n < a.T ? a.targets[n] : -1;
  }

  int pos = 0;
  for (int ti = t_begin; ti < t_end; ++ti) {
    while (ti >= a.st.tile0[pos + 1]) ++pos;
    const int r0 = (ti - a.st.tile0[pos]) * BM;
    const int rows = min(BM, a.st.rows[pos] - r0);
    const int64_t gid0 = a.st.off[pos] + r0;
    const S* Wt = (const S*)a.st.w[pos] + (int64_t)r0 * a.d;

    f32x16_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
    G::run(acc, Wt, a.d, 0, rows, (const S*)a.H, a.d, n0, (int)a.T, a.d, smem);

    const bool full = rows == BM;
    const int lim = rows - wm - 4 * (lane >> 5);
    fold_tile<MB, NB>(acc, full, lim, m_run, s_run);
#pragma unroll
    for (int j = 0; j < NB; ++j)
      gather_target<MB, NB>(acc, j, tgt[j] - gid0, rows, wm, lane, a.y_tgt,
                            n0 + wn + 32 * j + (lane & 31));
  }
  write_partials<G>(a, m_run, s_run, split, n0, (float*)smem);
}

// The forward on small tiles (see Ring): the slices of a workgroup's whole range of
// vocabulary tiles form one stream through the ring.  The token blocks of one vocabulary
// range run side by side on an XCD, so that its L2 reads their W once.
template <class E, class G>
__global__ void __launch_bounds__(G::NT, G::OCC* G::NWAVES / 4) stream_fwd_kernel(FwdArgs a) {
  using S = typename E::storage;
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB;
  __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = G::wave_m(wave), wn = G::wave_n(wave);
  const int logical = xcd_logical(blockIdx.x, gridDim.x);
  const int split = logical / a.n_tok_blocks;
  const int n0 = (logical % a.n_tok_blocks) * BN;
  const int t_begin = (int)((int64_t)split * a.n_tiles / a.n_splits);
  const int t_end = (int)((int64_t)(split + 1) * a.n_tiles / a.n_splits);

  float m_run[NB], s_run[NB];
  int64_t tgt[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    m_run[j] = kNoLogit;
    s_run[j] = 0.f;
    const int64_t n = n0 + wn + 32 * j + (lane & 31);
    tgt[j] = n < a.T ? a.targets[n] : -1;
  }
  // (waited for here: from now on only slice loads, and rare stores, are in flight)
#pragma unroll
  for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(tgt[j]));

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int nk = (a.d + G::BK - 1) / G::BK;
  const int tail_chunks = a.d % G::BK ? a.d % G::BK / E::VEC : G::CPR;
  const int total = (t_end - t_begin) * nk;

  // the loading side of the stream: tile, slice and ring slot of the next slice to load
  const char* baseB = (const char*)((const S*)a.H + (int64_t)n0 * a.d);
  const char* baseA = nullptr;
  uint32_t offA[G::A_LOADS], offB[G::B_LOADS];
  G::offsets(offB, (int)min((int64_t)BN, a.T - n0), a.d, wave, lane);
  int l_pos = 0, l_tile = t_begin, l_kt = 0, l_slot = 0, loaded = 0;
  auto load_next = [&]() {
    if (l_kt == 0) {
      while (l_tile >= a.st.tile0[l_pos + 1]) ++l_pos;
      const int r0 = (l_tile - a.st.tile0[l_pos]) * BM;
      baseA = (const char*)((const S*)a.st.w[l_pos] + (int64_t)r0 * a.d);
      G::offsets(offA, min(BM, a.st.rows[l_pos] - r0), a.d, wave, lane);
    }
    const int chunks = l_kt == nk - 1 ? tail_chunks : G::CPR;
    const uint32_t l = lds0 + (uint32_t)(l_slot * G::SLICE_BYTES);
    G::issue(baseA + (int64_t)l_kt * 128, offA, chunks, l, wave, lane);
    G::issue(baseB + (int64_t)l_kt * 128, offB, chunks, l + BM * 128, wave, lane);
    if (++l_kt == nk) {
      l_kt = 0;
      ++l_tile;
    }
    l_slot = l_slot + 1 == G::STAGES ? 0 : l_slot + 1;
    ++loaded;
  };
  for (int k = 0; k < min(G::STAGES - 1, total); ++k) load_next();

  f32x16_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
  int pos = 0, ti = t_begin, kt = 0, slot = 0;
  for (int it = 0; it < total; ++it) {
    // Slice `it` has landed (loads return in order; all but the youngest STAGES - 2
    // slices are waited for, at the end of the stream all of them), and no wave reads
    // the slot refilled next any more.
    if (loaded - it == G::STAGES - 1)
      wait_vmcnt<(G::STAGES - 2) * G::NLOADS>();
    else
      wait_vmcnt<0>();
    wait_lgkmcnt0();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (loaded < total) load_next();
    __builtin_amdgcn_sched_barrier(0);
    G::multiply(acc, smem + slot * G::SLICE_BYTES, wm, wn, lane);
    slot = slot + 1 == G::STAGES ? 0 : slot + 1;
    if (++kt == nk) {
      kt = 0;
      while (ti >= a.st.tile0[pos + 1]) ++pos;
      const int r0 = (ti - a.st.tile0[pos]) * BM;
      const int rows = min(BM, a.st.rows[pos] - r0);
      const int64_t gid0 = a.st.off[pos] + r0;
      const bool full = rows == BM;
      const int lim = rows - wm - 4 * (lane >> 5);
      fold_tile<MB, NB>(acc, full, lim, m_run, s_run);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        gather_target<MB, NB>(acc, j, tgt[j] - gid0, rows, wm, lane, a.y_tgt,
                              n0 + wn + 32 * j + (lane & 31));
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i][j] = f32x16_t{};
      }
      ++ti;
    }
  }
  write_partials<G>(a, m_run, s_run, split, n0, (float*)smem);
}

// Folds the per-split partial states of each token, then finalises lse = m + log z and loss = lse - y_target.
template <int LPT>
__global__ void __launch_bounds__(256) comb_kernel(CombArgs a) {
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPT;
  if (t >= a.T) return;
  float m, s;
  merge_splits<LPT>(a.m_part, a.s_part, a.T, t, a.n_splits, m, s);
  if (threadIdx.x % LPT) return;
  const float lse = (m + __builtin_amdgcn_logf(s)) * kLn2;
  const int64_t tg = a.targets[t];
  float loss;
  if (tg == a.ignore_index) {
    loss = 0.f;
  } else if (tg < 0 || tg >= a.V) {
    loss = __builtin_nanf("");
    atomicAdd(a.bad_counter, 1ull);
  } else {
    loss = lse - a.y_tgt[t];
  }
  a.lse[t] = lse;
  a.loss[t] = loss;
}

// Per-shard fold (one meeting of Algorithm 2 for a state that travels with the
// activations).  The state's m plane is kept in natural units so that it can be
// exchanged as plain numbers; the kernels work in the base-2 domain.
__global__ void __launch_bounds__(256) state_init_kernel(float* state, int64_t T) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= T) return;
  state[t] = -INFINITY;
  state[T + t] = 0.f;
  state[2 * T + t] = 0.f;
}

// state (m, s) <- fold of state and the shard's split partials.
template <int LPT>
__global__ void __launch_bounds__(256) fold_merge_kernel(FoldArgs a) {
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPT;
  if (t >= a.T) return;
  float mq, sq;
  merge_splits<LPT>(a.m_part, a.s_part, a.T, t, a.n_splits, mq, sq);
  if (threadIdx.x % LPT) return;
  const float m_in = a.state[t];
  float m = m_in == -INFINITY ? -INFINITY : m_in * kLog2e;
  float s = a.state[a.T + t];
  merge_state(m, s, mq, sq);
  a.state[t] = m == -INFINITY ? -INFINITY : m * kLn2;
  a.state[a.T + t] = s;
}

// lse = m + log s and loss = lse - y (0 when ignored, NaN and counted when the
// target is outside [0, V)).
__global__ void __launch_bounds__(256) fold_finalize_kernel(FinArgs a) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= a.T) return;
  const float lse = a.state[t] + __builtin_amdgcn_logf(a.state[a.T + t]) * kLn2;
  const int64_t tg = a.targets[t];
  float loss;
  if (tg == a.ignore_index) {
    loss = 0.f;
  } else if (tg < 0 || tg >= a.V) {
    loss = __builtin_nanf("");
    atomicAdd(a.bad_counter, 1ull);
  } else {
    loss = lse - a.state[2 * a.T + t];
  }
  a.lse[t] = lse;
  a.loss[t] = loss;
}


// yt[t] = h_t . w_{targets[t]} (float32 sum of the exact products), one wavefront per
// token, 16-byte loads (d is a multiple of 8).  Targets outside [0, V) (ignored or out
// of range) give 0; the residual tiles do not use it for them.
template <class S>
__global__ void __launch_bounds__(256) target_logit_kernel(TgtArgs a) {
  constexpr int VEC = 16 / (int)sizeof(S);
  if (a.count && blockIdx.x == 0) {
    __shared__ int bad[256];
    int n = 0;
    for (int64_t i = threadIdx.x; i < a.T; i += 256) {
      const int64_t tg = a.targets[i];
      n += tg != a.ignore_index && (tg < 0 || tg >= a.V);
    }
    bad[threadIdx.x] = n;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
      if ((int)threadIdx.x < o) bad[threadIdx.x] += bad[threadIdx.x + o];
      __syncthreads();
    }
    if (threadIdx.x == 0) *a.count = (unsigned long long)bad[0];
  }
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (t >= a.T) return;
  const int64_t tg = a.targets[t];
  float acc = 0.f;
  if (tg >= 0 && tg < a.V) {
    int p = 0;
    while (p + 1 < a.st.P && !(tg >= a.st.off[p] && tg < a.st.off[p] + a.st.rows[p])) ++p;
    const S* w = (const S*)a.st.w[p] + (tg - a.st.off[p]) * (int64_t)a.d;
    const S* h = (const S*)a.H + t * (int64_t)a.d;
    for (int k = lane * VEC; k < a.d; k += 64 * VEC) {
      const uint4 hv = *(const uint4*)(h + k), wv = *(const uint4*)(w + k);
      if constexpr (sizeof(S) == 2) {
        const uint32_t hh[4] = {hv.x, hv.y, hv.z, hv.w}, ww[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          acc = __builtin_fmaf(__uint_as_float(hh[q] << 16), __uint_as_float(ww[q] << 16), acc);
          acc = __builtin_fmaf(__uint_as_float(hh[q] & 0xFFFF0000u), __uint_as_float(ww[q] & 0xFFFF0000u), acc);
        }
      } else {
        acc = __builtin_fmaf(__uint_as_float(hv.x), __uint_as_float(wv.x), acc);
        acc = __builtin_fmaf(__uint_as_float(hv.y), __uint_as_float(wv.y), acc);
        acc = __builtin_fmaf(__uint_as_float(hv.z), __uint_as_float(wv.z), acc);
        acc = __builtin_fmaf(__uint_as_float(hv.w), __uint_as_float(wv.w), acc);
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o);
  if (lane == 0) a.yt[t] = acc;
}

// Counts out-of-range targets of a token range (backward's copy of the check).
__global__ void count_bad_kernel(const int64_t* targets, int64_t T, int64_t V, int64_t ignore_index,
                                 unsigned long long* counter) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (t < T) {
    const int64_t tg = targets[t];
    if (tg != ignore_index && (tg < 0 || tg >= V)) atomicAdd(counter, 1ull);
  }
}

__global__ void __launch_bounds__(256) sum_parts_kernel(const float4* __restrict__ part, int n,
                                                        int64_t len, float4* __restrict__ out) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < len; i += stride) {
    float4 s = part[i];
#pragma unroll 4
    for (int k = 1; k < n; ++k) {
      const float4 v = part[(int64_t)k * len + i];
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
    out[i] = s;
  }
}

// out = in^T in the k-blocked layout: in is row-major [R][ld_in]; out is
// [R_pad / KB][C][KB] with KB = 128 / sizeof(S) (element (c, r) at
// ((r / KB) C + c) KB + r % KB), zero for R <= r < R_pad.  One 64 x 64 tile per
// workgroup (one-dimensional grid, row blocks fastest: T / 64 up to 2^17 and
// d / 64 up to 2^16 exceed a grid dimension), staged through LDS with 16-byte
// accesses to global memory on both sides.  A tile row of 64 elements is VPR
// 16-byte vectors; vector v of tile row i sits in slot v ^ ((i / VEC) % VPR), so
// that the column reads of the store side (VEC consecutive rows of one column
// per lane, rows VEC g .. VEC g + VEC - 1 for lane group g) fall in distinct
// banks.  Needs C, ld_in and both base addresses in whole 16-byte vectors and
// R_pad a multiple of KB (checked by run_transpose).
template <class S>
__global__ void __launch_bounds__(256) transpose_kernel(TransposeArgs a) {
  constexpr int VEC = 16 / (int)sizeof(S);  // elements per 16-byte vector
  constexpr int VPR = 64 / VEC;             // vectors per tile row
  constexpr int ROWS = 256 / VPR;           // tile rows (or output rows) per pass
  constexpr int KB = 128 / (int)sizeof(S);
  __shared__ __attribute__((aligned(16))) S tile[64][64];
  const S* in = (const S*)a.in;
  S* out = (S*)a.out;
  const uint32_t n_rb = ((uint32_t)a.R_pad + 63u) / 64u;
  const int r0 = (int)(blockIdx.x % n_rb) * 64, c0 = (int)(blockIdx.x / n_rb) * 64;
  const int v = threadIdx.x % VPR, i0 = threadIdx.x / VPR;
#pragma unroll
  for (int i = i0; i < 64; i += ROWS) {
    const int r = r0 + i, c = c0 + VEC * v;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (r < a.R && c < a.C) x = *(const uint4*)(in + (int64_t)r * a.ld_in + c);
    *(uint4*)&tile[i][(v ^ ((i / VEC) % VPR)) * VEC] = x;
  }
  __syncthreads();
  // lane group g = v gathers tile rows VEC g .. VEC g + VEC - 1 of one column
#pragma unroll
  for (int cl = i0; cl < 64; cl += ROWS) {
    const int c = c0 + cl, r = r0 + VEC * v;
    if (c < a.C && r < a.R_pad) {
      union {
        uint4 u;
        S e[VEC];
      } y;
#pragma unroll
      for (int j = 0; j < VEC; ++j) y.e[j] = tile[VEC * v + j][((cl / VEC) ^ v) * VEC + cl % VEC];
      *(uint4*)(out + ((int64_t)(r / KB) * a.C + c) * KB + r % KB) = y.u;
    }
  }
}


template <class E, class G>
static bool launch_fwd_g(const FwdArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n_tok_blocks * a.n_splits);
  hipLaunchKernelGGL((fwd_kernel<E, G>), dim3(grid), dim3(G::NT), 0, s, a);
  return launched_ok();
}
template <class E, class G>
static bool launch_stream(const FwdArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.n_tok_blocks * a.n_splits);
  hipLaunchKernelGGL((stream_fwd_kernel<E, G>), dim3(grid), dim3(G::NT), 0, s, a);
  return launched_ok();
}
template <class E>
static bool launch_fwd(const FwdArgs& a, hipStream_t s) {
  switch (a.kind) {
    case 1: return launch_stream<E, typename Cfg<E>::Stream128>(a, s);
    case 2: return launch_stream<E, typename Cfg<E>::Stream64>(a, s);
  }
  if (a.d % E::KB == 0) return launch_fwd_g<E, typename Cfg<E>::Logits>(a, s);
  return launch_fwd_g<E, typename Cfg<E>::LogitsTail>(a, s);
}

// ---------------------------------------------------------------------------
// Library-owned forward workspace for callers that cannot allocate (see
// vp_ce_forward_noalloc).  Each device the library runs on holds its own copy
// from the first use until the process ends.  In host code `scratch` names a
// host-side stand-in, not device memory: its device address is looked up once
// per device with hipGetSymbolAddress, and only that address is ever passed on.
static __device__ __align__(256) unsigned char scratch[kScratchBytes];

namespace {
constexpr int kMaxDevices = 64;
std::mutex scratch_mu;
void* scratch_addr[kMaxDevices] = {};
}  // namespace

bool scratch_base(void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return false;
  std::lock_guard<std::mutex> lock(scratch_mu);
  if (!scratch_addr[dev]) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return false;
    scratch_addr[dev] = p;
  }
  *out = scratch_addr[dev];
  return true;
}

// ---- entry points used by the host API (vpce_api.cpp) ----
TileShape tile_shape(int dtype) {
  using L = Cfg<Bf16>::Logits;
  static_assert(L::BM == Cfg<F32>::Logits::BM && L::BN == Cfg<F32>::Logits::BN, "one large tile");
  return TileShape{L::BM, L::BN, dtype == 1 ? Bf16::KB : F32::KB};
}

// Microseconds a workgroup takes per 128-byte slice of one tile, measured on launches
// that fill the chip: with two or more token blocks sharing W in the L2s, and with one
// block, where W streams from memory (bfloat16, d = 4096 and 1000, T = 40..1024; float32
// is bound by its matrix rate either way, d = 2880).
template <class E>
static FwdTile fwd_tile_of(int kind) {
  constexpr bool b16 = sizeof(typename E::storage) == 2;
  using G0 = typename Cfg<E>::Logits;
  using G1 = typename Cfg<E>::Stream128;
  using G2 = typename Cfg<E>::Stream64;
  switch (kind) {
    case 1: return b16 ? FwdTile{G1::BM, G1::BN, G1::OCC, 1.4, 1.5} : FwdTile{G1::BM, G1::BN, G1::OCC, 4.44, 4.44};
    case 2: return b16 ? FwdTile{G2::BM, G2::BN, G2::OCC, 0.47, 0.5} : FwdTile{G2::BM, G2::BN, G2::OCC, 1.33, 1.36};
  }
  return b16 ? FwdTile{G0::BM, G0::BN, G0::OCC, 1.4, 1.8} : FwdTile{G0::BM, G0::BN, G0::OCC, 7.45, 7.45};
}
FwdTile fwd_tile(int dtype, int kind) {
  return dtype == 1 ? fwd_tile_of<Bf16>(kind) : fwd_tile_of<F32>(kind);
}

int bwd_col_blocks(int cls, int d) {
  using B = Cfg<Bf16>;
  return cls == 1   ? col_blocks<B::Tr128x64, B::Tr128x64>(d).n
         : cls == 2 ? col_blocks<B::Tr128, B::Tr128>(d).n
                    : col_blocks<B::Tr256, B::Tr320>(d).n;
}
// The tiles have the same shapes for both types.
BwdTile bwd_tile(int dtype, int cls) {
  using B = Cfg<Bf16>;
  const bool b16 = dtype == 1;
  switch (cls) {
    case 1: return BwdTile{B::Tr128x64::BM, B::Tr128x64::BN, b16 ? 0.34 : 1.0};
    case 2: return BwdTile{B::Tr128::BM, B::Tr128::BN, b16 ? 0.55 : 1.88};
    case 3: return BwdTile{B::Mm::BM, B::Mm::BN, b16 ? 1.38 : 6.9};
  }
  return BwdTile{B::Tr256::BM, B::Tr256::BN, 1.40};
}
bool run_stage(int dtype, int cls, const StageArgs& a, hipStream_t s) {
  if (a.grad_entropy) return run_stage_entropy(dtype, cls, a, s);
  return dtype == 1 ? launch_stage<Bf16, false>(cls, a, s) : launch_stage<F32, false>(cls, a, s);
}
bool run_sum_parts(const float* part, int n, int64_t len, float* out, hipStream_t s) {
  const int64_t vecs = len / 4, blocks = std::min<int64_t>((vecs + 255) / 256, 2048);
  hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)blocks), dim3(256), 0, s, (const float4*)part, n,
                     vecs, (float4*)out);
  return launched_ok();
}

bool run_ws_init(unsigned long long* counter, hipStream_t s) {
  hipLaunchKernelGGL(ws_init_kernel, dim3(1), dim3(64), 0, s, counter);
  return launched_ok();
}
bool run_fill_zero(float* p, int64_t n, hipStream_t s) {
  if (n <= 0) return true;
  const int64_t blocks = std::min<int64_t>((n + 255) / 256, 4096);
  hipLaunchKernelGGL(fill_zero_kernel, dim3((unsigned)blocks), dim3(256), 0, s, p, n);
  return launched_ok();
}
bool run_fwd(int dtype, const FwdArgs& a, hipStream_t s) {
  return dtype == 1 ? launch_fwd<Bf16>(a, s) : launch_fwd<F32>(a, s);
}
bool run_comb(const CombArgs& a, hipStream_t s) {
  if (a.n_splits >= kManySplits)
    hipLaunchKernelGGL(comb_kernel<16>, dim3((unsigned)((a.T + 15) / 16)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(comb_kernel<1>, dim3((unsigned)((a.T + 255) / 256)), dim3(256), 0, s, a);
  return launched_ok();
}
bool run_state_init(float* state, int64_t T, hipStream_t s) {
  if (T <= 0) return true;
  hipLaunchKernelGGL(state_init_kernel, dim3((unsigned)((T + 255) / 256)), dim3(256), 0, s, state, T);
  return launched_ok();
}
bool run_fold_merge(const FoldArgs& a, hipStream_t s) {
  if (a.T <= 0) return true;
  if (a.n_splits >= kManySplits)
    hipLaunchKernelGGL(fold_merge_kernel<16>, dim3((unsigned)((a.T + 15) / 16)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(fold_merge_kernel<1>, dim3((unsigned)((a.T + 255) / 256)), dim3(256), 0, s, a);
  return launched_ok();
}
bool run_fold_finalize(const FinArgs& a, hipStream_t s) {
  if (a.T <= 0) return true;
  hipLaunchKernelGGL(fold_finalize_kernel, dim3((unsigned)((a.T + 255) / 256)), dim3(256), 0, s, a);
  return launched_ok();
}
bool run_count_bad(const int64_t* targets, int64_t T, int64_t V, int64_t ignore_index,
                   unsigned long long* counter, hipStream_t s) {
  if (T <= 0) return true;
  hipLaunchKernelGGL(count_bad_kernel, dim3((unsigned)((T + 255) / 256)), dim3(256), 0, s, targets,
                     T, V, ignore_index, counter);
  return launched_ok();
}
bool run_target_logits(int dtype, const TgtArgs& a, hipStream_t s) {
  if (a.T <= 0) return true;
  const dim3 grid((unsigned)((a.T + 3) / 4));
  if (dtype == 1)
    hipLaunchKernelGGL(target_logit_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(target_logit_kernel<float>, grid, dim3(256), 0, s, a);
  return launched_ok();
}
bool run_transpose(int dtype, const TransposeArgs& a, hipStream_t s) {
  if (a.C <= 0 || a.R_pad <= 0) return true;
  const int esz = dtype == 1 ? 2 : 4, vec = 16 / esz, kb = 128 / esz;
  // the 16-byte accesses of the kernel: whole vectors on both sides, whole k-blocks
  if (a.C % vec != 0 || a.ld_in % vec != 0 || a.R_pad % kb != 0 || a.R < 0 || a.R > a.R_pad ||
      ((uintptr_t)a.in & 15u) != 0 || ((uintptr_t)a.out & 15u) != 0)
    return false;
  const int64_t blocks = (int64_t)((a.R_pad + 63) / 64) * ((a.C + 63) / 64);
  if (blocks > 0x7fffffff) return false;  // beyond any operand that fits in memory
  const dim3 grid((unsigned)blocks);
  if (dtype == 1)
    hipLaunchKernelGGL(transpose_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(transpose_kernel<float>, grid, dim3(256), 0, s, a);
  return launched_ok();
}

}  // namespace vpce
