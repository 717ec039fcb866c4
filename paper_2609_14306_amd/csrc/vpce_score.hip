// Scoring of tokens, for gfx950 (MI355X): the forward of the vocabulary projection (see
// vpce_kernels.hip) with the entropy of every token and its most likely ids, in bfloat16, float32
// and 8-bit floating point.
//
// Entropy.  With the running maximum m and d = y - m, the fold keeps r = sum e^d - 1, without the maximum's own
// term, and u = sum e^d d; where m grows by c, the whole old sum 1 + r goes into r' = e^-c (1 + r) and u' = e^-c
// (u - c (1 + r)).  Then
//   lse = m + log(1 + r),   entropy = lse - sum p y = log(1 + r) - u / (1 + r),
// two terms that are not negative, each to float32's relative precision: of a token of which one id holds all but
// 1e-7 the entropy is right to 8e-6 of itself (sum e^d itself would lose 1e-7 to the 1 beside it).  Summing
// the rest apart and exact distances take two instructions an element: T = 4096, d = 2880, V = 201088 in bfloat16
// 1.1%, T = 8192, d = 7168, V = 129280 in 8 bits nothing, narrow rows (T = 8192, d = 512, V = 50000) 5%.
//
// Alternatives.  No logits are kept; the fold leaves the maximum of every four consecutive ids
// (fine) and of the logits that a lane holds of a tile (coarse).  The K + 2 largest fine maxima,
// ties by the lower ids, hold the K largest logits but for what the product's sums round: the logits of
// those ids are taken again in float64, where the products of the operands are exact, and ranked by
// that.  Where the maxima come nearer to the last one given than eight times what the ones looked at are
// off by, or than a rule for sums of d terms (run_top), all that do are looked at, up to 64: an answer differs from the
// float64 one only where more lie that near, or a sum is off by more (1 to 2 us of a call).
//
// 8-bit operands (e4m3) have a power of two as scale for every 128 columns of a token and every 128
// x 128 block of a shard.  A slice of 128 bytes is one such block: the matrix instruction of
// 64 columns takes the scales as its own operands, for nothing.  It adds eight products of a row
// with bits below 2^-13 of the largest one's power of two cut off, and such sums in float32 (as
// measured; the instruction without scales and the 16 x 16 ones are the same): a logit is off by 1.5e-5
// of the logits' spread.  Over many ids that averages out; where a few hold the probability it does not
// (logits of spread 4: entropies 1e-5 off).  So the ids with a probability of 2^-7 and more have their
// exact logits put into lse and entropy behind the fold (top_kernel, kHeavy): 1e-7 to 8e-7 then.  That
// takes the maxima also without alternatives (T = 8192, d = 7168, V = 129280 6% of the time, half of it that
// kernel's).  Widened to bfloat16, where the products are exact, few tokens took 164 us instead of 132 (T = 1 to 64,
// V = 151936, d = 4096), with one wavefront a SIMD 137 (T to 32) and 183, and large tiles would run at half the rate.
//
// What bounds it (kernels alone).  Many tokens: the matrix rate at the clock that the chip's power
// leaves: T = 4096, d = 2880, V = 201088 in bfloat16 3.65 ms (1301 TFLOP/s, as vp_ce_forward; 3.87 and 0.23 for the
// ranking with 8 alternatives), T = 8192, d = 7168, V = 129280 in 8 bits 5.58 ms (2720) and 0.19, T = 1000, d = 7168,
// V = 32000 in float32 3.36 ms (136).  Few tokens: reading W: T = 1, d = 4096, V = 151936 in bfloat16 226 us (208 at
// best, 6.0 TB/s) and 31 for 20 alternatives, T = 40 in 8 bits 131 us (117 at best, 5.3 TB/s) and 21 for 5.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "vpce_internal.h"
#include "vpce_lanes.h"
#include "vpce_tiles.h"

namespace vpce {

// 8-bit elements: a 128-byte slice row is 128 columns, one scale.
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
struct F8 {
  using storage = uint8_t;
  using frag16 = i32x4_t;
  static constexpr int VEC = 16, KB = 128;
  // 64 columns: a lane holds 32 of them, two 16-byte chunks, the same ones in both operands.
  __device__ static i32x8_t join(frag16 x, frag16 y) {
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ static f32x16_t mma(i32x8_t a, i32x8_t b, f32x16_t c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
  }
};
template <class E>
constexpr bool kIsF8 = sizeof(typename E::storage) == 1;

// Scales in LDS: of the BN tokens of a workgroup, [nb][BN], and of as many of its vocabulary
// tiles as have room, [tile][128-row block][nb].
template <class G>
struct Scales {
  static constexpr int BLOCKS = G::BM / 128;
  static constexpr int H_BYTES = G::BN * kF8MaxBlocks;
  static constexpr int W_BYTES = (160 * 1024 - G::LDS_ELEMS - H_BYTES) / 16 * 16;
  static_assert(W_BYTES >= BLOCKS * kF8MaxBlocks, "one tile's scales");
  uint8_t *h, *w;
  int nb, first, count;  // tiles whose scales are there

  __device__ __forceinline__ void load_tokens(const ScoreArgs& a, int n0) {
    nb = a.nb;
    first = count = 0;
    for (int i = threadIdx.x; i < G::BN * nb; i += G::NT) {
      const int64_t n = n0 + i / nb;
      h[(i % nb) * G::BN + i / nb] = a.h_scale[(n < a.f.T ? n : a.f.T - 1) * nb + i % nb];
    }
  }
  // Scales of the tiles from ti on, before end; all threads, and no other is between barriers.
  __device__ __forceinline__ void load_tiles(const ScoreArgs& a, int ti, int end) {
    first = ti;
    count = min(end - ti, W_BYTES / (BLOCKS * nb));
    __syncthreads();
    for (int i = threadIdx.x; i < count * BLOCKS * nb; i += G::NT) {
      const int b = i / nb, tile = ti + b / BLOCKS;
      int pos = 0;
      while (tile >= a.f.st.tile0[pos + 1]) ++pos;
      const int row = (tile - a.f.st.tile0[pos]) * BLOCKS + b % BLOCKS;
      const int rows = (a.f.st.rows[pos] + 127) / 128;
      w[i] = a.w_scale[pos][(int64_t)min(row, rows - 1) * nb + i % nb];
    }
    __syncthreads();
  }
  __device__ __forceinline__ bool has(int ti) const { return ti >= first && ti < first + count; }
  __device__ __forceinline__ int of_rows(int ti, int wm, int kt) const {
    return w[((ti - first) * BLOCKS + wm / 128) * nb + kt];
  }
  __device__ __forceinline__ int of_token(int column, int kt) const { return h[kt * G::BN + column]; }
};

struct NoScales {};
template <class E, class G>
using ScalesFor = std::conditional_t<kIsF8<E>, Scales<G>, NoScales>;

// The 256 x 256 tile of GemmDma for 8-bit operands: its slices, swizzle and loads, two sub-steps
// of 64 columns a slice.  All loads of slice kt + 2 go out during the second sub-step of slice kt,
// one behind each of its first MFMAs, and have the first sub-step of slice kt + 1 to land.
template <bool KTAIL_>
struct GemmF8 : GemmDma<256, 256, 2, 4, F8, KTAIL_> {
  using Base = GemmDma<256, 256, 2, 4, F8, KTAIL_>;
  using typename Base::F16;
  using typename Base::Loads;
  using typename Base::S;
  using Base::BK, Base::KTAIL, Base::MB, Base::NB, Base::NLOADS, Base::NM, Base::STAGES;
  using Base::issue_one, Base::plan, Base::read_one, Base::slot_bytes, Base::wait_slices;

  __device__ __forceinline__ static void run(f32x16_t (&acc)[MB][NB], const S* __restrict__ A, int64_t lda,
                                             int M, const S* __restrict__ B, int64_t ldb, int n0, int N, int K,
                                             char* smem, const Scales<GemmF8>& sc, int ti) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = Base::wave_m(wave), wn = Base::wave_n(wave);
    const int nk = (K + BK - 1) / BK;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    Loads L;
    plan(L, A, lda, 0, M, B, ldb, n0, N, wave, lane);
    L.kblkA = L.kblkB = BK;
    if constexpr (KTAIL) {
      L.tail_kt = K % BK ? nk - 1 : -1;
      L.tail_chunks = K % BK / F8::VEC;
    }
    const int pro = min(STAGES, nk);
    for (int kt = 0; kt < pro; ++kt)
#pragma unroll
      for (int q = 0; q < NLOADS; ++q) issue_one(L, kt, q, lds0, wave);
    wait_slices(pro - 1);
    __builtin_amdgcn_s_barrier();
    const char* ring = smem;
    // fragment idx (A's row blocks, then B's) of the sub-step that begins with chunks 2 kk
    auto read = [&](const char* slot, int kk, int idx) {
      return F8::join(read_one(slot, wm, wn, kk, lane, idx), read_one(slot, wm, wn, kk + 1, lane, idx));
    };
    i32x8_t a[MB], b[2][NB];
    int sa, sb[NB], sa_next, sb_next[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) a[i] = read(ring, 0, i);
#pragma unroll
    for (int j = 0; j < NB; ++j) b[0][j] = read(ring, 0, MB + j);
    sa_next = sc.of_rows(ti, wm, 0);
#pragma unroll
    for (int j = 0; j < NB; ++j) sb_next[j] = sc.of_token(wn + 32 * j + (lane & 31), 0);
    for (int kt = 0; kt < nk; ++kt) {
      sa = sa_next;
#pragma unroll
      for (int j = 0; j < NB; ++j) sb[j] = sb_next[j];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const char* src;
        int skk;
        if (kk == 0) {
          src = ring + slot_bytes(kt);
          skk = 2;
          const int next = min(kt + 1, nk - 1);
          sa_next = sc.of_rows(ti, wm, next);
#pragma unroll
          for (int j = 0; j < NB; ++j) sb_next[j] = sc.of_token(wn + 32 * j + (lane & 31), next);
        } else {
          // as in GemmDma::run: slice kt + 1 has landed, and on the last slice a spare barrier
          wait_vmcnt<0>();
          wait_lgkmcnt0();
          __builtin_amdgcn_s_barrier();
          src = ring + slot_bytes(kt + 1);
          skk = 0;
        }
        const bool loads = kk == 1 && kt + STAGES < nk;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int idx = 0; idx < NM; ++idx) {
          const int i = idx / NB, jj = idx % NB, j = (i & 1) ? NB - 1 - jj : jj;
          // (a wave in its products goes before the other one of its SIMD: 1.1% of T = 8192, d = 7168)
          if (idx == 0) __builtin_amdgcn_s_setprio(1);
          acc[i][j] = F8::mma(a[i], b[kk][j], acc[i][j], sa, sb[j]);
          if (idx == NM - 1) __builtin_amdgcn_s_setprio(0);
          // (an empty statement that keeps the product in front of the branches around the loads:
          // the compiler would move all sixteen of a slice behind them)
          asm volatile("" : "+v"(acc[i][j]));
          __builtin_amdgcn_sched_barrier(0);
          if (idx < NB) b[kk ^ 1][idx] = read(src, skk, MB + idx);
          if (jj == NB - 1) a[i] = read(src, skk, i);
          if (loads && idx < NLOADS) issue_one(L, kt + STAGES, idx, lds0, wave);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    wait_vmcnt<0>();
    wait_lgkmcnt0();
    __builtin_amdgcn_s_barrier();
  }
  static_assert(NLOADS <= NM, "one load behind each MFMA");
};

// The streamed tiles of Ring for 8-bit operands: 64 tokens, and 128 from 65 on, where the small tile
// would read W twice and the large one leaves half of itself and of its third round empty (T = 128, d =
// 4096, V = 151936: 180 us without, 140 so).
template <int BN_, int STAGES_>
struct RingF8 : Ring<128, BN_, 4, 2, STAGES_, F8> {
  using Base = Ring<128, BN_, 4, 2, STAGES_, F8>;
  using typename Base::F16;
  using Base::BM, Base::MB, Base::NB, Base::key;
  __device__ __forceinline__ static void multiply(f32x16_t (&acc)[MB][NB], const char* slot, int wm, int wn,
                                                  int lane, int sa, const int (&sb)[NB]) {
#pragma unroll
    for (int kk = 0; kk < 4; kk += 2) {
      auto read = [&](int first, int r) {
        const char* row = slot + (first + r) * 128;
        const int chunk = 2 * kk + (lane >> 5);
        return F8::join(*(const F16*)(row + ((chunk ^ key(r)) << 4)), *(const F16*)(row + (((chunk + 2) ^ key(r)) << 4)));
      };
      i32x8_t fa[MB], fb[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) fa[i] = read(0, wm + 32 * i + (lane & 31));
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[j] = read(BM, wn + 32 * j + (lane & 31));
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = F8::mma(fa[i], fb[j], acc[i][j], sa, sb[j]);
    }
  }
};

// ---------------------------------------------------------------------------
// A lane's state of a token: the maximum m, r = sum e^(y - m) - 1 and u = sum e^(y - m) (y - m).  The term
// of the maximum itself is exactly 1 and is not in r, so that a small rest keeps its digits.  An empty state
// has m = kNoLogit, whose e^(y - m) is 0 beside any logit, and r = -1, the sum 0, where it leaves the workgroup.
struct Fold {
  float m, r, u;
};
constexpr float kLeast = -1e4f;  // e^kLeast is 0: the distance that farther maxima are held to
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// The state with the maximum `m` in place of its own, which is no larger: its whole sum is part of r then.
__device__ __forceinline__ Fold rescaled(Fold f, float m) {
  const float c = fmaxf(f.m - m, kLeast), e = exp_of(c), s = 1.f + f.r;
  return Fold{m, s * e, e * __builtin_fmaf(c, s, f.u)};
}
__device__ __forceinline__ void merge_fold(Fold& f, Fold o) {
  const bool first = f.m >= o.m;
  const Fold hi = first ? f : o, lo = rescaled(first ? o : f, hi.m == -INFINITY ? 0.f : hi.m);
  f = Fold{hi.m, hi.r + lo.r, hi.u + lo.u};
}

// Tokens whose fine maxima lie side by side: on the large tiles the 32 of a column block, so that
// every store fills whole lines of memory (T = 4096, V = 201088: the stores cost the product 1% and
// the pieces of 16 bytes that a token alone has 3.7%), and one on the small ones, which have few
// tokens (T = 1, V = 151936: 261 us in all, and 265 with 32).
template <class G>
constexpr int kFineTokens = G::SKIPS ? 32 : 1;

// Folds column block j of a logits tile (fold_tile of vpce_tiles.h with the third sum) and, with
// TOP, leaves its maxima: fine, the bm / 4 ones of this tile and the lane's token, and coarse
// (both null for a token that does not exist).  Rows from `lim` on are minus infinity.
template <int MB, int NB, bool TOP, int TOK>
__device__ __forceinline__ void fold_score(f32x16_t (&acc)[MB][NB], int j, bool full, int lim, Fold& f,
                                           int lane, float* fine, float* coarse) {
  float g[MB][4], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x16_t& v = acc[i][j];
      g[i][q] = fmaxf(fmaxf(v[4 * q], v[4 * q + 1]), fmaxf(v[4 * q + 2], v[4 * q + 3]));
      top = fmaxf(top, g[i][q]);
    }
  }
  if constexpr (TOP) {
    if (coarse) *coarse = top;
    if (!full)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) g[i][q] = 32 * i + 8 * q < lim ? g[i][q] : __builtin_nanf("");
    if constexpr (TOK == 32) {
      if (fine)
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) fine[(8 * i + 2 * q + (lane >> 5)) * 32] = g[i][q];
    } else {
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        // The lanes l and l + 32 hold the even and the odd ones of the block's eight maxima; after
        // two swaps of half wavefronts they hold the first and the last four.
        typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
        const u32x2_t x = __builtin_bit_cast(
            u32x2_t, __builtin_amdgcn_permlane32_swap(__float_as_uint(g[i][0]), __float_as_uint(g[i][2]), false, false));
        const u32x2_t y = __builtin_bit_cast(
            u32x2_t, __builtin_amdgcn_permlane32_swap(__float_as_uint(g[i][1]), __float_as_uint(g[i][3]), false, false));
        if (fine)
          *(float4*)(fine + 8 * i + 4 * (lane >> 5)) =
              make_float4(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(y[0]), __uint_as_float(y[1]));
      }
    }
  }
  const float m = fmaxf(f.m, top);
  // s - rest are the terms of 1 (the maximum, and what equals it): rest leaves them out, and keeps its digits.
  float s, rest, u;
  for (bool low = !full;; low = true) {
    // e^d d of a logit of minus infinity is 0, not 0 times infinity.  Where there is one, as in the dead rows of a
    // shard's last tile, they are raised to a distance whose e^d is 0, too (a maximum with every d costs 1%).
    if (low) {
      const float least = fmaxf(m - fmaxf(2000.f, __builtin_fabsf(m)), kNoLogit);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = acc[i][j][r] < least ? least : acc[i][j][r];
    }
    s = rest = u = 0.f;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      if (i > 0) __builtin_amdgcn_sched_barrier(0);  // (16 exponents at a time: more of them are spilled)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float d = acc[i][j][r] - m, e = exp_of(d);
        s += e;
        rest += __builtin_amdgcn_fractf(e);
        u = __builtin_fmaf(e, d, u);
      }
      // (the sums are made here: the compiler would hold all exponentials for them until the loop's end)
      asm volatile("" : "+v"(s), "+v"(rest), "+v"(u));
    }
    if (low || !__any(u != u)) break;
  }
  const bool rises = m > f.m;  // one of the terms of 1 is the new maximum
  if (rises) f = rescaled(f, m);
  f.r = f.r + rest + (rintf(s - rest) - (rises ? 1.f : 0.f));
  f.u += u;
}

// Folds a tile: rows past the end of its shard (all but the last tile have none) become minus
// infinity, 2^x of which is 0, so that one loop without masks serves both.
template <class G, bool TOP>
__device__ __forceinline__ void fold_block(const ScoreArgs& a, f32x16_t (&acc)[G::MB][G::NB], int ti, int rows, int n0,
                                           int wm, int wn, int lane, Fold (&f)[G::NB]) {
  constexpr int TOK = kFineTokens<G>;
  const bool full = rows == G::BM;
  const int lim = rows - wm - 4 * (lane >> 5);
  if (!full)
#pragma unroll
    for (int j = 0; j < G::NB; ++j)
#pragma unroll
      for (int i = 0; i < G::MB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          acc[i][j][r] = 32 * i + 8 * (r >> 2) + (r & 3) < lim ? acc[i][j][r] : -INFINITY;
#pragma unroll
  for (int j = 0; j < G::NB; ++j) {
    const int64_t n = n0 + wn + 32 * j + (lane & 31);
    float *fine = nullptr, *coarse = nullptr;
    if (TOP && n < a.f.T) {
      fine = a.fine + (((int64_t)ti * ((a.f.T + TOK - 1) / TOK) + n / TOK) * (G::BM / 4) + wm / 4) * TOK + n % TOK;
      coarse = a.coarse + ((int64_t)ti * a.f.T + n) * (2 * G::WGM) + wm / G::WM * 2 + (lane >> 5);
    }
    fold_score<G::MB, G::NB, TOP, TOK>(acc, j, full, lim, f[j], lane, fine, coarse);
  }
}

// End of a workgroup: as write_partials of vpce_tiles.h, with the third plane.
template <class G>
__device__ __forceinline__ void write_folds(const ScoreArgs& a, Fold (&f)[G::NB], int split, int n0, float* red) {
  constexpr int BN = G::BN, NB = G::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = G::wave_n(wave);
#pragma unroll
  for (int j = 0; j < NB; ++j)
    merge_fold(f[j], Fold{__shfl_xor(f[j].m, 32), __shfl_xor(f[j].r, 32), __shfl_xor(f[j].u, 32)});
  __syncthreads();
  const int wr = wave / G::WGN;  // red: [WGM][3][BN]
  if (lane < 32) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float* r = red + wr * 3 * BN + wn + 32 * j + lane;
      r[0] = f[j].m;
      r[BN] = f[j].r;
      r[2 * BN] = f[j].u;
    }
  }
  __syncthreads();
  if (wr == 0 && lane < 32) {
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int c = wn + 32 * j + lane;
      for (int w = 1; w < G::WGM; ++w) {
        const float* r = red + w * 3 * BN + c;
        merge_fold(f[j], Fold{r[0], r[BN], r[2 * BN]});
      }
      const int64_t n = n0 + c;
      if (n < a.f.T) {
        const bool none = f[j].m == kNoLogit;
        a.f.m_part[(int64_t)split * a.f.T + n] = none ? -INFINITY : f[j].m;
        a.f.s_part[(int64_t)split * a.f.T + n] = none && f[j].r >= 0.f ? -1.f : f[j].r;  // (or NaN)
        a.u_part[(int64_t)split * a.f.T + n] = f[j].u;
      }
    }
  }
}

// fwd_kernel of vpce_kernels.hip with the fold above.
template <class E, class G, bool TOP>
__global__ void __launch_bounds__(G::NT, G::OCC) score_kernel(ScoreArgs a) {
  using S = typename E::storage;
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB;
  constexpr int RING = G::LDS_ELEMS * (int)sizeof(S);
  __shared__ __attribute__((aligned(16))) char smem[kIsF8<E> ? 160 * 1024 : RING];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = G::wave_m(wave), wn = G::wave_n(wave);
  const int logical = xcd_logical(blockIdx.x, gridDim.x);
  const int tb = logical / a.f.n_splits;
  const int split = logical % a.f.n_splits;
  const int n0 = tb * BN;
  const int t_begin = (int)((int64_t)split * a.f.n_tiles / a.f.n_splits);
  const int t_end = (int)((int64_t)(split + 1) * a.f.n_tiles / a.f.n_splits);

  Fold f[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) f[j] = Fold{kNoLogit, -1.f, 0.f};
  ScalesFor<E, G> sc;
  if constexpr (kIsF8<E>) {
    sc.h = (uint8_t*)smem + RING;
    sc.w = sc.h + Scales<G>::H_BYTES;
    sc.load_tokens(a, n0);
  }
  int pos = 0;
  for (int ti = t_begin; ti < t_end; ++ti) {
    while (ti >= a.f.st.tile0[pos + 1]) ++pos;
    const int r0 = (ti - a.f.st.tile0[pos]) * BM;
    const int rows = min(BM, a.f.st.rows[pos] - r0);
    const S* Wt = (const S*)a.f.st.w[pos] + (int64_t)r0 * a.f.d;

    f32x16_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
    if constexpr (kIsF8<E>) {
      if (!sc.has(ti)) sc.load_tiles(a, ti, t_end);
      G::run(acc, Wt, a.f.d, rows, (const S*)a.f.H, a.f.d, n0, (int)a.f.T, a.f.d, smem, sc, ti);
    } else {
      G::run(acc, Wt, a.f.d, 0, rows, (const S*)a.f.H, a.f.d, n0, (int)a.f.T, a.f.d, (S*)smem);
    }
    fold_block<G, TOP>(a, acc, ti, rows, n0, wm, wn, lane, f);
  }
  write_folds<G>(a, f, split, n0, (float*)smem);
  if (blockIdx.x == 0 && tid == 0 && a.f.counter) *a.f.counter = 0ull;
}

// stream_fwd_kernel of vpce_kernels.hip with the fold above.
template <class E, class G, bool TOP>
__global__ void __launch_bounds__(G::NT, G::OCC* G::NWAVES / 4) score_stream_kernel(ScoreArgs a) {
  using S = typename E::storage;
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB;
  __shared__ __attribute__((aligned(16))) char smem[kIsF8<E> ? 160 * 1024 : G::LDS_BYTES];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = G::wave_m(wave), wn = G::wave_n(wave);
  const int logical = xcd_logical(blockIdx.x, gridDim.x);
  const int split = logical / a.f.n_tok_blocks;
  const int n0 = (logical % a.f.n_tok_blocks) * BN;
  const int t_begin = (int)((int64_t)split * a.f.n_tiles / a.f.n_splits);
  const int t_end = (int)((int64_t)(split + 1) * a.f.n_tiles / a.f.n_splits);

  Fold f[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) f[j] = Fold{kNoLogit, -1.f, 0.f};
  ScalesFor<E, G> sc;
  if constexpr (kIsF8<E>) {
    sc.h = (uint8_t*)smem + G::LDS_BYTES;
    sc.w = sc.h + Scales<G>::H_BYTES;
  }

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int nk = (a.f.d + G::BK - 1) / G::BK;
  const int tail_chunks = a.f.d % G::BK ? a.f.d % G::BK / E::VEC : G::CPR;
  const int total = (t_end - t_begin) * nk;

  const char* baseB = (const char*)((const S*)a.f.H + (int64_t)n0 * a.f.d);
  const char* baseA = nullptr;
  uint32_t offA[G::A_LOADS], offB[G::B_LOADS];
  G::offsets(offB, (int)min((int64_t)BN, a.f.T - n0), a.f.d, wave, lane);
  int l_pos = 0, l_tile = t_begin, l_kt = 0, l_slot = 0, loaded = 0;
  auto load_next = [&]() {
    if (l_kt == 0) {
      while (l_tile >= a.f.st.tile0[l_pos + 1]) ++l_pos;
      const int r0 = (l_tile - a.f.st.tile0[l_pos]) * BM;
      baseA = (const char*)((const S*)a.f.st.w[l_pos] + (int64_t)r0 * a.f.d);
      G::offsets(offA, min(BM, a.f.st.rows[l_pos] - r0), a.f.d, wave, lane);
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
  if constexpr (kIsF8<E>) {  // (while the first slices are on their way)
    sc.load_tokens(a, n0);
    sc.load_tiles(a, t_begin, t_end);
  }

  f32x16_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
  int pos = 0, ti = t_begin, kt = 0, slot = 0;
  for (int it = 0; it < total; ++it) {  // (the waits of stream_fwd_kernel)
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
    if constexpr (kIsF8<E>) {
      const int sa = sc.of_rows(ti, wm, kt);
      int sb[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) sb[j] = sc.of_token(wn + 32 * j + (lane & 31), kt);
      G::multiply(acc, smem + slot * G::SLICE_BYTES, wm, wn, lane, sa, sb);
    } else {
      G::multiply(acc, smem + slot * G::SLICE_BYTES, wm, wn, lane);
    }
    slot = slot + 1 == G::STAGES ? 0 : slot + 1;
    if (++kt == nk) {
      kt = 0;
      while (ti >= a.f.st.tile0[pos + 1]) ++pos;
      const int r0 = (ti - a.f.st.tile0[pos]) * BM;
      const int rows = min(BM, a.f.st.rows[pos] - r0);
      fold_block<G, TOP>(a, acc, ti, rows, n0, wm, wn, lane, f);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i][j] = f32x16_t{};
      }
      ++ti;
      if constexpr (kIsF8<E>)
        if (ti < t_end && !sc.has(ti)) sc.load_tiles(a, ti, t_end);
    }
  }
  write_folds<G>(a, f, split, n0, (float*)smem);
  if (blockIdx.x == 0 && tid == 0 && a.f.counter) *a.f.counter = 0ull;
}

// Operands in float64, where their products are exact: the N elements of 16 bytes.
template <class E>
struct Dot;
template <>
struct Dot<Bf16> {
  static constexpr int N = 8;
  static constexpr uint32_t MAGNITUDE = 0x7fff7fffu;
  __device__ static void unpack(uint4 u, double (&f)[N]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[2 * k] = (double)__uint_as_float(w[k] << 16);
      f[2 * k + 1] = (double)__uint_as_float(w[k] & 0xffff0000u);
    }
  }
};
template <>
struct Dot<F32> {
  static constexpr int N = 4;
  static constexpr uint32_t MAGNITUDE = 0x7fffffffu;
  __device__ static void unpack(uint4 u, double (&f)[N]) {
    f[0] = (double)__uint_as_float(u.x);
    f[1] = (double)__uint_as_float(u.y);
    f[2] = (double)__uint_as_float(u.z);
    f[3] = (double)__uint_as_float(u.w);
  }
};
template <>
struct Dot<F8> {
  static constexpr int N = 16;
  static constexpr uint32_t MAGNITUDE = 0x7f7f7f7fu;
  __device__ static void unpack(uint4 u, double (&f)[N]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false);
      const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
      f[4 * k] = (double)lo[0];
      f[4 * k + 1] = (double)lo[1];
      f[4 * k + 2] = (double)hi[0];
      f[4 * k + 3] = (double)hi[1];
    }
  }
};
__device__ __forceinline__ double pow2_byte(int b) {  // 2^(b - 127), NaN for 255
  return b == 255 ? __builtin_nan("") : ldexp(1.0, b - 127);
}

// A wavefront finishes a token: joins its splits as comb_kernel of vpce_kernels.hip does, with the
// entropy, which is NaN where lse is not finite; returns lse.  The target's logit is taken here, in
// float64, and not from the tile that has it: the matrix unit rounds an 8-bit product's sum more
// coarsely than a float32 one (2e-5 of a logit, d = 4096), which lse averages over the vocabulary and
// a single logit does not (loss off by 2.8e-6 relative with the tile's, 6e-8 so); and a wave of the
// product's kernel keeps no targets in registers that it needs for operands.
struct Finished {
  float lse, entropy;
  double y;  // the target's logit
  int64_t target;
};
template <class E>
__device__ __forceinline__ Finished finish_token(const ScoreCombArgs& a, const ScoreArgs& sa, int64_t t, int lane) {
  using S = typename E::storage;
  constexpr int N = Dot<E>::N;
  const int64_t tg = a.c.targets[t];
  Fold f{-INFINITY, -1.f, 0.f};
#pragma unroll 4
  for (int k = lane; k < a.c.n_splits; k += 64) {
    const int64_t i = (int64_t)k * a.c.T + t;
    merge_fold(f, Fold{a.c.m_part[i], a.c.s_part[i], a.u_part[i]});
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
    merge_fold(f, Fold{__shfl_xor(f.m, o), __shfl_xor(f.r, o), __shfl_xor(f.u, o)});
  const float log_s = log1pf(f.r), lse = f.m + log_s;
  double y = 0.0;
  if (tg >= 0 && tg < a.c.V) {
    const ShardTable& st = sa.f.st;
    const int64_t end = lane < st.P ? st.off[lane] + st.rows[lane] : INT64_MAX;  // a shard a lane
    const int pos = __popcll(__ballot(end <= tg));
    const int64_t row = tg - st.off[pos];
    const uint4* h = (const uint4*)((const S*)sa.f.H + t * sa.f.d);
    const uint4* w = (const uint4*)((const S*)st.w[pos] + row * sa.f.d);
#pragma unroll 4
    for (int c = lane; c < sa.f.d / N; c += 64) {
      double x[N], v[N], p = 0.0, scale = 1.0;
      Dot<E>::unpack(h[c], x);
      Dot<E>::unpack(w[c], v);
      if constexpr (kIsF8<E>)
        scale = pow2_byte(sa.h_scale[t * sa.nb + c / 8]) * pow2_byte(sa.w_scale[pos][row / 128 * sa.nb + c / 8]);
#pragma unroll
      for (int k = 0; k < N; ++k) p = fma(x[k], v[k], p);
      y = fma(p, scale, y);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) y += __shfl_xor(y, o);
  }
  return Finished{lse, log_s - f.u / (1.f + f.r), y, tg};
}

// Its results, by one lane.
__device__ __forceinline__ void store_token(const ScoreCombArgs& a, int64_t t, const Finished& f) {
  float loss;
  if (f.target == a.c.ignore_index) {
    loss = 0.f;
  } else if (f.target < 0 || f.target >= a.c.V) {
    loss = __builtin_nanf("");
  } else {
    loss = (float)((double)f.lse - f.y);
  }
  a.c.lse[t] = f.lse;
  a.c.loss[t] = loss;
  if (a.entropy) a.entropy[t] = f.entropy;
}
__device__ __forceinline__ void count_target(const ScoreCombArgs& a, int64_t target) {
  if (target != a.c.ignore_index && (target < 0 || target >= a.c.V)) atomicAdd(a.c.bad_counter, 1ull);
}

template <class E>
__global__ void __launch_bounds__(256) score_comb_kernel(ScoreCombArgs a, ScoreArgs sa) {
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.c.T) return;
  const Finished f = finish_token<E>(a, sa, t, threadIdx.x & 63);
  if (threadIdx.x & 63) return;
  store_token(a, t, f);
  count_target(a, f.target);
}

// ---------------------------------------------------------------------------
// The most likely ids of a token, one workgroup of NT threads each, which finishes the token too.
// Bound by latency for few tokens (a few dependent reads of maxima, then four rows of W for each group
// of ids that is looked at; 16 wavefronts side by side), and for many by those rows: (K + 2) 4 d
// elements a token.  Of the 30 us of T = 1, d = 4096, K = 20 in bfloat16 3 are the threshold, 2 the groups, 13 the
// rows in two turns, most of it their conversion to float64 (units of two rows, which convert h twice, took
// 6 more), and 3 the order.  Comparisons of all with all go a lane each, counted by ballots: one thread
// for each of 88 logits took 5 us longer.
constexpr int kExtra = 2, kGroupRoom = 64;
static_assert(VP_MAX_TOP + kExtra <= kGroupRoom, "groups of a token");
constexpr int kCoarseRoom = 512, kFineRoom = 1024;
// 8-bit operands: the ids with a probability of 2^-7 and more have their part in lse and in the entropy
// exactly.  A logit is off by 1.5e-5 of the logits' spread, which the rest of the ids averages out: with
// random logits of spread 4 entropies are off by 8e-7 relative, and 1.2e-5 without.
constexpr float kHeavy = -7.f * 0.6931471805599453f;
constexpr int kKeep = 4;  // fours of coarse maxima that a thread keeps in registers

// The larger logit first, the lower id among equals.
template <class V, class I>
__device__ __forceinline__ bool before(V va, I ia, V vb, I ib) {
  return va > vb || (va == vb && ia < ib);
}

// (Many tokens in bfloat16: five wavefronts a SIMD, for which it is held to 102 registers, T = 4096 0.24 -> 0.22 ms;
// 8 bits would spill.)
template <class E, int NT>
__global__ void __launch_bounds__(NT, NT == 256 && sizeof(typename E::storage) == 2 ? 5 : 1) top_kernel(TopArgs a) {
  using S = typename E::storage;
  constexpr int N = Dot<E>::N, WAVES = NT / 64;
  constexpr int UNROLL = NT != 1024 ? 2 : kIsF8<E> ? 1 : 4;  // of a row's chunks (a lane of 1024 has 128 registers)
  __shared__ float side[WAVES][64];
  __shared__ float cand_v[kFineRoom];
  __shared__ int cand_g[kFineRoom], list[kCoarseRoom];
  __shared__ int sel[kGroupRoom];
  __shared__ float sel_v[kGroupRoom];
  __shared__ double val[4 * kGroupRoom], last_s;
  __shared__ int64_t gid[4 * kGroupRoom];
  __shared__ unsigned off_s;
  __shared__ int count[2];
  __shared__ float tau_s, lse_s;
  __shared__ float best_v[WAVES];
  __shared__ int best_g[WAVES];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const FwdArgs& f = a.s.f;
  const int64_t T = f.T, t = xcd_logical(blockIdx.x, gridDim.x);
  int64_t* ids = a.ids + t * a.top;
  float* loss = a.loss + t * a.top;
  const int F = a.bm / 4, cpt = a.cpt, fpc = F / cpt, n4 = f.n_tiles * (cpt / 4);
  const int want = a.top + kExtra;
  // coarse maxima 4 c .. 4 c + 3, and fine maximum g of all tiles
  const int per_tile = cpt / 4, shift = per_tile - 1;  // 1 or 2 fours a tile
  auto coarse = [&](int c) {
    return ((const float4*)a.s.coarse)[((int64_t)(c >> shift) * T + t) * per_tile + (c & shift)];
  };
  const int tok = a.tok;
  const float* fine_t = a.s.fine + t / tok * F * tok + t % tok;
  auto fine = [&](int g) { return fine_t[((int64_t)(g / F) * ((T + tok - 1) / tok) * F + g % F) * tok]; };
  auto max4 = [](float4 v) { return fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)); };

  // (without alternatives, of 8-bit operands, none are selected here)
  const bool any = !kIsF8<E> || a.top > 0;
  int groups = 0, n = 0;
  if (any) {
    // tau: the want-th largest of 64 maxima over the threads' shares, which as many coarse maxima
    // reach
    const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    float4 keep[kKeep];
    float mine = -INFINITY;
#pragma unroll
    for (int k = 0; k < kKeep; ++k) keep[k] = tid + k * NT < n4 ? coarse(tid + k * NT) : none;
#pragma unroll
    for (int k = 0; k < kKeep; ++k) mine = fmaxf(mine, max4(keep[k]));
#pragma unroll 8
    for (int c = tid + kKeep * NT; c < n4; c += NT) mine = fmaxf(mine, max4(coarse(c)));
    side[wave][lane] = mine;
    if (tid < 2) count[tid] = 0;
    __syncthreads();
    if (wave == 0) {
      float all = mine;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) all = fmaxf(all, side[w][lane]);
      int rank = 0;
#pragma unroll
      for (int k = 0; k < 64; ++k) rank += before(lane_read(all, k), k, all, lane);
      if (rank == want - 1) tau_s = all;
    }
    __syncthreads();
    const float tau = tau_s;
    // The fine maxima that reach tau, or with `above` lie above it, among cand_*; whether they fit.
    auto collect = [&](bool above) {
      auto in = [&](float x) { return above ? x > tau : x >= tau; };
      auto take = [&](int c, float4 v) {
        const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (in(x[j])) {
            const int k = atomicAdd(&count[0], 1);
            if (k < kCoarseRoom) list[k] = 4 * c + j;
          }
      };
      if (in(mine)) {
#pragma unroll
        for (int k = 0; k < kKeep; ++k)
          if (tid + k * NT < n4) take(tid + k * NT, keep[k]);
        for (int c = tid + kKeep * NT; c < n4; c += NT) take(c, coarse(c));
      }
      __syncthreads();
      const int n_coarse = count[0];
      if (n_coarse > kCoarseRoom) return false;
      for (int e = tid; e < n_coarse * fpc; e += NT) {
        const int c = list[e / fpc], within = c % cpt;
        const int g = c / cpt * F + (within >> 1) * 2 * fpc + 2 * (e % fpc) + (within & 1);
        const float v = fine(g);
        if (in(v)) {
          const int k = atomicAdd(&count[1], 1);
          if (k < kFineRoom) {
            cand_v[k] = v;
            cand_g[k] = g;
          }
        }
      }
      __syncthreads();
      return count[1] <= kFineRoom;
    };
    bool fits = collect(false), tied = false;
    if (!fits) {
      // Many logits equal tau (a token of zeros has nothing else): those above it, and of the equal
      // ones the first.
      __syncthreads();
      if (tid < 2) count[tid] = 0;
      __syncthreads();
      tied = fits = collect(true);
    }
    n = count[1];
    if (fits) {
      groups = min(n, want);
      for (int e = wave; e < n; e += WAVES) {  // (a lane compares with every 64th other one)
        const float v = cand_v[e];
        const int g = cand_g[e];
        int r = 0;
        for (int k = 0; k < n; k += 64) {
          const int o = min(k + lane, n - 1);
          r += __popcll(__ballot(k + lane < n && before(cand_v[o], cand_g[o], v, g)));
        }
        if (r < want && lane == 0) {
          sel[r] = g;
          sel_v[r] = v;
        }
      }
      for (int base = 0; tied && groups < want && base < f.n_tiles * F; base += NT) {
        const int g = base + tid;
        const uint64_t hit = __ballot(g < f.n_tiles * F && fine(min(g, f.n_tiles * F - 1)) == tau);
        if (lane == 0) best_g[wave] = __popcll(hit);
        __syncthreads();
        int at = groups + __popcll(hit & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          at += w < wave ? best_g[w] : 0;
          groups += best_g[w];
        }
        if (hit >> lane & 1 && at < want) {
          sel[at] = g;
          sel_v[at] = tau;
        }
        __syncthreads();
      }
      groups = min(groups, want);
    } else {
      // More above tau than there is room for (they lie in few threads' shares): the groups one by one,
      // each the next in order after the one before.
      float last_v = INFINITY;
      int last_g = -1;
      for (; groups < want; ++groups) {
        float v = -INFINITY;
        int g = INT32_MAX;
        for (int k = tid; k < f.n_tiles * F; k += NT) {
          const float x = fine(k);
          if (x == x && before(last_v, last_g, x, k) && before(x, k, v, g)) {
            v = x;
            g = k;
          }
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const float vo = __shfl_xor(v, o);
          const int go = __shfl_xor(g, o);
          if (before(vo, go, v, g)) {
            v = vo;
            g = go;
          }
        }
        if (lane == 0) {
          best_v[wave] = v;
          best_g[wave] = g;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
          if (before(best_v[w], best_g[w], v, g)) {
            v = best_v[w];
            g = best_g[w];
          }
        __syncthreads();
        if (g == INT32_MAX) break;
        if (tid == 0) {
          sel[groups] = g;
          sel_v[groups] = v;
        }
        last_v = v;
        last_g = g;
      }
    }
  }
  const int chunks = f.d / N;
  if (tid == 0) {
    off_s = 0;
    last_s = -INFINITY;
  }
  __syncthreads();
  Finished token;
  if (wave == 0) {
    token = finish_token<E>(a.comb, a.s, t, lane);
    if (lane == 0) {
      lse_s = token.lse;
      if (!kIsF8<E>) store_token(a.comb, t, token);
      count_target(a.comb, token.target);
    }
  }
  for (bool again = false;; again = true) {
    for (int s = wave - 1; s < groups && wave > 0; s += WAVES - 1) {
      const int g = __builtin_amdgcn_readfirstlane(sel[s]), tile = g / F;
      const int pos = __popcll(__ballot(f.st.tile0[lane + 1] <= tile));  // (a shard a lane)
      const int row = (tile - f.st.tile0[pos]) * a.bm + g % F * 4, live = min(4, f.st.rows[pos] - row);
      const uint4* w = (const uint4*)((const S*)f.st.w[pos] + (int64_t)row * f.d);
      // (H's row goes through an empty statement: the compiler would hold it for all groups in registers)
      const uint4* h = (const uint4*)((const S*)f.H + t * f.d);
      asm volatile("" : "+s"(h));
      double acc[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll UNROLL
      for (int c = lane; c < chunks; c += 64) {
        double x[N], y[N];
        uint4 raw[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) raw[r] = w[(int64_t)min(r, live - 1) * chunks + c];
        Dot<E>::unpack(h[c], x);
        double scale = 1.0;
        if constexpr (kIsF8<E>) {
          const int b = c / (128 / N);
          scale = pow2_byte(a.s.h_scale[t * a.s.nb + b]) * pow2_byte(a.s.w_scale[pos][(int64_t)(row / 128) * a.s.nb + b]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          Dot<E>::unpack(raw[r], y);
          double p = 0.0;
#pragma unroll
          for (int k = 0; k < N; ++k) p = fma(x[k], y[k], p);
          acc[r] = fma(p, scale, acc[r]);
        }
      }
      // the four sums over the lanes: two of them to each half of the wavefront, then one to each quarter
      const bool up = lane & 32, odd = lane & 16;
      double two[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) two[r] = (up ? acc[2 + r] : acc[r]) + __shfl_xor(up ? acc[r] : acc[2 + r], 32);
      double v = (odd ? two[1] : two[0]) + __shfl_xor(odd ? two[0] : two[1], 16);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o);
      const int r = lane >> 4;
      if ((lane & 15) == 0) {
        val[4 * s + r] = v;
        gid[4 * s + r] = r < live ? f.st.off[pos] + row + r : -1;
      }
      // what the float32 maximum is off by
      double most = r < live ? v : -INFINITY;
      most = fmax(most, __shfl_xor(most, 16));
      most = fmax(most, __shfl_xor(most, 32));
      const float off = (float)__builtin_fabs(most - (double)sel_v[s]);
      if (lane == 0 && off < INFINITY) atomicMax(&off_s, __float_as_uint(off));
    }
    __syncthreads();
    float lse = lse_s;
    if (!(__builtin_fabsf(lse) < INFINITY)) {
      if (tid < a.top) {
        ids[tid] = -1;
        loss[tid] = __builtin_nanf("");
      }
      if (kIsF8<E> && tid == 0) store_token(a.comb, t, token);
      return;
    }
    const float heavy = lse + kHeavy;
    if constexpr (kIsF8<E>) {
      // With the matrix unit's m and the exact m + c of the largest id of a group, p = e^z, z = m - lse:
      //   A = sum p (e^c - 1),  B = sum p ((e^c - 1) (z + c) + c),
      //   lse' = lse + log(1 + A),  entropy' = (entropy - B) / (1 + A) + log(1 + A).
      if (wave == 0) {
        const float m = lane < groups ? sel_v[lane] : -INFINITY;
        float z = 0.f, c = 0.f, p = 0.f;
        if (m >= heavy) {
          double most = -INFINITY;
          for (int r = 0; r < 4; ++r) most = gid[4 * lane + r] >= 0 ? fmax(most, val[4 * lane + r]) : most;
          z = m - lse;
          c = (float)(most - (double)m);
          p = expf(z);
        }
        float far = __builtin_fabsf(c), up = p > 0.f ? z + c : 0.f;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          far = fmaxf(far, __shfl_xor(far, o));
          up = fmaxf(up, __shfl_xor(up, o));
        }
        // (c far from 0, of operands with a few products above all others: the sums themselves, over e^up)
        const bool small = far < 0.5f;
        const float e = small ? expm1f(c) : expf(z + c - up);
        float A = p * e, B = p * __builtin_fmaf(e, z + c, c), P = p, Q = p * z;
        if (!small) {
          A = p > 0.f ? e : 0.f;
          B = p > 0.f ? e * (z + c) : 0.f;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          A += __shfl_xor(A, o);
          B += __shfl_xor(B, o);
          P += __shfl_xor(P, o);
          Q += __shfl_xor(Q, o);
        }
        Finished exact = token;
        if (small) {
          const float l = log1pf(A);
          exact.lse += l;
          exact.entropy = fmaxf((token.entropy - B) / (1.f + A) + l, 0.f);
        } else {
          const float mass = 1.f - P > 1e-6f ? 1.f - P : 0.f, rest = expf(-up), all = mass * rest + A, l = up + logf(all);
          exact.lse += l;
          exact.entropy = fmaxf(l - ((mass > 0.f ? fminf(-token.entropy - Q, 0.f) * rest : 0.f) + B) / all, 0.f);
        }
        if (lane == 0) {
          best_v[0] = exact.lse;
          store_token(a.comb, t, exact);
        }
      }
      __syncthreads();
      lse = best_v[0];
    }
    n = 4 * groups;
    int live = 0;
    for (int k = 0; k < n; k += 64) live += __popcll(__ballot(k + lane < n && gid[min(k + lane, n - 1)] >= 0));
    for (int e = wave; e < n; e += WAVES) {
      const double v = val[e];
      const int64_t g = gid[e];
      if (g < 0) continue;
      int r = 0;
      for (int k = 0; k < n; k += 64) {
        const int o = min(k + lane, n - 1);
        r += __popcll(__ballot(k + lane < n && gid[o] >= 0 && before(val[o], gid[o], v, g)));
      }
      if (r < a.top && lane == 0) {
        ids[r] = g;
        loss[r] = (float)((double)lse - v);
        if (r == a.top - 1) last_s = v;
      }
    }
    // fewer ids than asked for
    if (tid >= live && tid < a.top) {
      ids[tid] = -1;
      loss[tid] = INFINITY;
    }
    if (again || (any && groups < want)) return;
    // A group that is not among them has a float32 maximum of sel_v[want - 1] at most, and one id of it a
    // logit that is larger by what the sums are off by, for which eight times the most that was seen stands, and
    // a.sum_off of the logit at least: the ones seen may be exact.  Where that reaches the last logit that is given,
    // all groups that could are looked at, if there is room; and so are those that the sums above should have.
    // (A token of zeros has exact logits, all equal.)
    __syncthreads();
    const float least = any ? sel_v[want - 1] : INFINITY;
    float near = INFINITY;
    const double last = last_s, margin = fmax(8.0 * (double)__uint_as_float(off_s), a.sum_off * __builtin_fabs(last));
    if (a.top > 0 && (double)least + margin >= last && last > -INFINITY) {
      uint32_t bits = 0;  // of H's row, but for signs
#pragma unroll 1
      for (int c = tid; c < chunks; c += NT) {
        const uint4 h = ((const uint4*)((const S*)f.H + t * f.d))[c];
        bits |= (h.x | h.y | h.z | h.w) & Dot<E>::MAGNITUDE;
      }
      if (__syncthreads_or((int)bits)) near = __double2float_rd(last - margin);
    }
    const float likely = kIsF8<E> && least >= heavy ? heavy : INFINITY;
    // (one of the two lists holds the other; where the longer one has no room the shorter one may)
    float border = fminf(near, likely), other = fmaxf(near, likely);
    for (;; border = other, other = INFINITY) {
      if (border == INFINITY) return;
      __syncthreads();
      if (tid < 2) count[tid] = 0;
      __syncthreads();
#pragma unroll 1
      for (int c = tid; c < n4; c += NT) {
        const float4 v = coarse(c);
#pragma unroll 1
        for (int j = 0; j < 4 && max4(v) >= border; ++j) {
          const int k = (j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w) >= border ? atomicAdd(&count[0], 1) : kCoarseRoom;
          if (k < kCoarseRoom) list[k] = 4 * c + j;
        }
      }
      __syncthreads();
      const int n_coarse = count[0];
      if (n_coarse > kCoarseRoom) continue;
#pragma unroll 1
      for (int e = tid; e < n_coarse * fpc; e += NT) {
        const int c = list[e / fpc], within = c % cpt;
        const int g = c / cpt * F + (within >> 1) * 2 * fpc + 2 * (e % fpc) + (within & 1);
        const float v = fine(g);
        const int k = v >= border ? atomicAdd(&count[1], 1) : kGroupRoom;
        if (k < kGroupRoom) {
          cand_v[k] = v;
          cand_g[k] = g;
        }
      }
      __syncthreads();
      n = count[1];
      if (n <= kGroupRoom) break;
    }
    if (n <= groups) return;
    groups = n;
    // (in their own order, not in the one that they came in: sums over them are the same bits every time)
    const int own = min(lane, n - 1), g = cand_g[own];
    const float v = cand_v[own];
    for (int k = wave; k < n; k += WAVES) {
      const float vk = lane_read(v, k);
      const int gk = __builtin_amdgcn_readlane(g, k), r = __popcll(__ballot(lane < n && before(v, g, vk, gk)));
      if (lane == 0) {
        sel[r] = gk;
        sel_v[r] = vk;
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
template <class E, class G>
static bool launch_score_g(const ScoreArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.f.n_tok_blocks * a.f.n_splits));
  if (kIsF8<E> || a.fine)
    hipLaunchKernelGGL((score_kernel<E, G, true>), grid, dim3(G::NT), 0, s, a);
  else if constexpr (!kIsF8<E>)
    hipLaunchKernelGGL((score_kernel<E, G, false>), grid, dim3(G::NT), 0, s, a);
  return launched_ok();
}
template <class E, class G>
static bool launch_score_stream(const ScoreArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.f.n_tok_blocks * a.f.n_splits));
  if (kIsF8<E> || a.fine)
    hipLaunchKernelGGL((score_stream_kernel<E, G, true>), grid, dim3(G::NT), 0, s, a);
  else if constexpr (!kIsF8<E>)
    hipLaunchKernelGGL((score_stream_kernel<E, G, false>), grid, dim3(G::NT), 0, s, a);
  return launched_ok();
}
// The tiles of the forward, but for float32, whose products are bound by their matrix rate down to 20
// tokens.  There two workgroups share a CU on all but the large tile: middle, the 128 x 128 tile of the
// backward; small, 128 x 64 with a ring of three slices; least, 128 x 32.  They reach 136, 134 and 107
// TFLOP/s (the large one 144) and leave shorter last rounds; the forward's tiles, of which one fits on a CU,
// reach 121 (256 x 128) and 101 (128 x 64).  d = 2880, V = 50000 in 4, microseconds with the forward's and with
// these: T = 1 248 / 139, T = 64 252 / 205, T = 128 386 / 373, T = 384 1163 / 912, T = 1024 2629 / 2344, T =
// 2048 4588 / 4440; d = 1000, V = 32003 in 5: T = 1333 806 / 760.
template <class E> struct ScoreCfg {
  using Large = typename Cfg<E>::Logits;
  using LargeTail = typename Cfg<E>::LogitsTail;
  using Small = typename Cfg<E>::Stream64;
  using Middle = typename Cfg<E>::Stream128;
};
template <> struct ScoreCfg<F8> {
  using Large = GemmF8<false>;
  using LargeTail = GemmF8<true>;
  using Small = RingF8<64, 6>;
  using Middle = RingF8<128, 4>;
};
template <> struct ScoreCfg<F32> {
  using Large = Cfg<F32>::Logits;
  using LargeTail = Cfg<F32>::LogitsTail;
  using Small = Cfg<F32>::Res128x64;
  using Middle = Cfg<F32>::Res128;
  using Least = Ring<128, 32, 4, 1, 3, F32>;
};
template <class E>
static bool launch_score(const ScoreArgs& a, hipStream_t s) {
  using C = ScoreCfg<E>;
  if (a.f.kind == 2) return launch_score_stream<E, typename C::Small>(a, s);
  if constexpr (sizeof(typename E::storage) == 4) {
    if (a.f.kind == 1) return launch_score_g<E, typename C::Middle>(a, s);
    if (a.f.kind == 3) return launch_score_stream<E, typename C::Least>(a, s);
  } else {
    if (a.f.kind == 1) return launch_score_stream<E, typename C::Middle>(a, s);
  }
  if (a.f.d % E::KB == 0) return launch_score_g<E, typename C::Large>(a, s);
  return launch_score_g<E, typename C::LargeTail>(a, s);
}

bool run_score(int dtype, const ScoreArgs& a, hipStream_t s) {
  if (dtype == VP_E4M3) return launch_score<F8>(a, s);
  return dtype == VP_BF16 ? launch_score<Bf16>(a, s) : launch_score<F32>(a, s);
}

template <class E>
static bool launch_comb(const ScoreCombArgs& a, const ScoreArgs& sa, hipStream_t s) {
  hipLaunchKernelGGL((score_comb_kernel<E>), dim3((unsigned)((a.c.T + 3) / 4)), dim3(256), 0, s, a, sa);
  return launched_ok();
}
bool run_score_comb(int dtype, const ScoreCombArgs& a, const ScoreArgs& sa, hipStream_t s) {
  return dtype == VP_BF16 ? launch_comb<Bf16>(a, sa, s) : launch_comb<F32>(a, sa, s);
}

// Microseconds per 128-byte slice, as in fwd_tile_of of vpce_kernels.hip.
FwdTile score_tile(int dtype, int kind) {
  if (dtype == VP_F32 && kind > 0) {
    using C = ScoreCfg<F32>;
    if (kind == 1) return FwdTile{C::Middle::BM, C::Middle::BN, C::Middle::OCC, 3.95, 3.95};
    if (kind == 2) return FwdTile{C::Small::BM, C::Small::BN, C::Small::OCC, 2.0, 2.2};
    return FwdTile{C::Least::BM, C::Least::BN, C::Least::OCC, 1.25, 1.5};
  }
  if (kind == 3) return FwdTile{0, 0, 0, 0.0, 0.0};
  if (dtype != VP_E4M3) return fwd_tile(dtype, kind);
  using C = ScoreCfg<F8>;
  if (kind == 0) return FwdTile{C::Large::BM, C::Large::BN, C::Large::OCC, 1.4, 1.8};
  if (kind == 1) return FwdTile{C::Middle::BM, C::Middle::BN, C::Middle::OCC, 0.7, 0.87};
  return FwdTile{C::Small::BM, C::Small::BN, C::Small::OCC, 0.47, 0.5};
}

// f of the tile that a problem runs on
template <class F>
static int of_tile(int dtype, int kind, F&& f) {
  using B = ScoreCfg<Bf16>;
  using C = ScoreCfg<F8>;
  using D = ScoreCfg<F32>;
  static_assert(B::Large::WGM == C::Large::WGM && B::Large::WGM == D::Large::WGM && B::Small::WGM == C::Small::WGM &&
                    B::Small::WGM == D::Small::WGM,
                "the types' tiles are alike");
  if (kind == 3) return f(D::Least{});
  if (kind == 1) return dtype == VP_F32 ? f(D::Middle{}) : dtype == VP_E4M3 ? f(C::Middle{}) : f(B::Middle{});
  return kind == 0 ? f(B::Large{}) : f(B::Small{});
}
int score_coarse(int dtype, int kind) {
  return of_tile(dtype, kind, [](auto g) { return 2 * decltype(g)::WGM; });
}

// Up to 512 tokens, two workgroups of 1024 a CU, the latency of a token counts.
template <class E>
static bool launch_top(TopArgs a, hipStream_t s) {
  // A float32 sum of d products has as many roundings at most, of partial sums of about its size, which mostly
  // cancel; the 8-bit products' cut is 1.5e-5.  Four times either.
  a.sum_off = kIsF8<E> ? 0x1p-14 : 0x1p-22 * std::sqrt((double)a.s.f.d);
  const dim3 grid((unsigned)a.s.f.T);
  if (a.s.f.T <= 512)
    hipLaunchKernelGGL((top_kernel<E, 1024>), grid, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((top_kernel<E, 256>), grid, dim3(256), 0, s, a);
  return launched_ok();
}
int score_tokens(int dtype, int kind) {
  return of_tile(dtype, kind, [](auto g) { return kFineTokens<decltype(g)>; });
}

bool run_top(int dtype, const TopArgs& a, hipStream_t s) {
  if (dtype == VP_E4M3) return launch_top<F8>(a, s);
  return dtype == VP_BF16 ? launch_top<Bf16>(a, s) : launch_top<F32>(a, s);
}

}  // namespace vpce
