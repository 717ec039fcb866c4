// The backward of the vocabulary projection: residual tiles, the contractions into dH and dW, and
// the launch that runs both (vpce_kernels.hip describes the whole).
#pragma once
#include "vpce_tiles.h"

namespace vpce {

// Byte offset of element (row, col) of a bfloat16 tile of ROWS rows staged in LDS as
// 64-column blocks of ROWS x 128 bytes, the 16-byte chunks of each row
// XOR-swizzled by (row / 2) % 8 so that the rows a write or read phase touches
// spread over the banks.  Each block is laid out exactly like the matching
// block of a k-blocked strip (32 KiB for 256 rows).
template <int ROWS>
__device__ __forceinline__ uint32_t tile_lds_byte(int row, int col) {
  return (uint32_t)((col >> 6) * (ROWS * 128) + row * 128 + ((((col & 63) >> 3) ^ ((row >> 1) & 7)) << 4) +
                    (col & 7) * 2);
}

// Copies the ROWS x COLS bfloat16 tile staged in LDS (see tile_lds_byte) to a
// k-blocked strip: block b (columns 64 b .. 64 b + 63) goes to the ROWS x 128 bytes at
// element ((kb0 + b) * rows_pitch + r0) * 64, one 16-byte chunk per thread and
// step, 1 KiB contiguous per wavefront store.
template <int NT, int ROWS, int COLS>
__device__ __forceinline__ void store_tile_blocked(const uint16_t* lds, uint16_t* __restrict__ dst,
                                                   uint32_t kb0, uint32_t rows_pitch, uint32_t r0) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int q = 0; q < ROWS * COLS / 8 / NT; ++q) {
    const int c = q * NT + tid;  // 16-byte chunk of the tile
    const int b = c / (ROWS * 8), row = (c >> 3) % ROWS, ch = c & 7;
    const uint4 v = *(const uint4*)((const char*)lds + b * (ROWS * 128) + row * 128 + ((ch ^ ((row >> 1) & 7)) << 4));
    *(uint4*)(dst + (((kb0 + (uint32_t)b) * rows_pitch + r0 + (uint32_t)row) * 64u + (uint32_t)ch * 8u)) = v;
  }
}

// Backward residual: recompute a logits tile of the (vocabulary chunk, token
// chunk) strip and store G = g (softmax - onehot) into the strip in both layouts:
// G[v][t] (token columns contiguous, for dW) and G^T[t][v] (vocabulary columns
// contiguous, for dH).  Rows and columns of the tile that fall outside the chunk
// are written as zeros so that both contractions can read whole 16-byte chunks
// past a ragged edge.
//
// Every element is first written as g p = sign(g) 2^(y log2e + log2|g| - lse log2e)
// (one multiply-add and one exponential: the upstream gradient is folded into the
// exponent, and an ignored token gets log2|g| = -inf, i.e. zeros); the one element
// of a token column that holds its target is then overwritten, by the one lane that
// owns it, with g (p_t - 1) computed in float32 from the token's target logit yt
// (a separate dot product; it agrees with the tile's own value up to float32
// summation order).  bfloat16 tiles go through LDS (free once the mainloop returns)
// once per layout, so that both layouts leave as whole 16-byte chunks, 1 KiB per
// wavefront store; the target elements are patched in LDS before each store.
//
// ENT: the loss has an entropy term, with the upstream gradient e of the token's entropy S =
// lse - sum_v p_v y_v.  dS / dy_v = -p_v (log p_v + S), so
//   G = g (p - onehot) - e p (log p + S) = p ((g - e S) - e log p) - g onehot,
// two multiply-adds, an exponential and a product per element with x = log2 p, which is held at
// kLeastLog2 from below: a logit of minus infinity has p = 0 and would give 0 * infinity.  An
// ignored token has g = 0 and keeps its entropy's term.
constexpr float kLeastLog2 = -1e4f;
template <class E, class G, bool ENT>
__device__ __forceinline__ void grad_tile(const GradArgs& a, const float* entropy, const float* grad_entropy,
                                          int vt, int tb, typename E::storage* smem) {
  using S = typename E::storage;
  constexpr int BM = G::BM, BN = G::BN, MB = G::MB, NB = G::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = G::wave_m(wave), wn = G::wave_n(wave);
  const int m0 = vt * BM, n0 = tb * BN;

  // The per-token inputs of this lane's token columns are loaded ahead of the
  // mainloop, which drains them with its own loads, so that their latency is not
  // paid after it.  Columns past the chunk read its last token (N >= 1 whenever a
  // residual tile runs) and are masked below.
  int64_t tgv[NB];
  float gv[NB], lsev[NB], ytv[NB], sv[NB], ev[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t t = a.t0 + min(n0 + wn + 32 * j + (lane & 31), a.N - 1);
    tgv[j] = a.targets[t];
    gv[j] = a.grad[t];
    lsev[j] = a.lse[t];
    ytv[j] = a.yt[t];
    sv[j] = ENT ? entropy[t] : 0.f;
    ev[j] = ENT ? grad_entropy[t] : 0.f;
  }

  f32x16_t acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x16_t{};
  G::run(acc, (const S*)a.W, a.d, m0, a.M, (const S*)a.H + a.t0 * a.d, a.d, n0, a.N, a.d, smem);
  // (keeps the compiler from moving arithmetic on the prefetched values, and the wait
  // it needs, in front of the mainloop)
#pragma unroll
  for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(tgv[j]), "+v"(gv[j]), "+v"(lsev[j]), "+v"(ytv[j]));
  if constexpr (ENT)
#pragma unroll
    for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(sv[j]), "+v"(ev[j]));

  // Strip offsets fit in 32 bits (the strip budget is capped below 2^31 elements).
  // Both strips are k-blocked (see GradArgs) with KB = E::KB elements per block.
  constexpr bool kBlocked = sizeof(S) == 2;  // bfloat16 tiles are staged through LDS
  constexpr uint32_t KB = E::KB;
  S* __restrict__ Gs = (S*)a.strip;
  S* __restrict__ Gt = (S*)a.strip_t;
  const uint32_t Tc = (uint32_t)a.Tc, Vc = (uint32_t)a.Vc;
  if constexpr (kBlocked) {
    static_assert(BM % 64 == 0 && BN % 64 == 0 && BM * BN % (8 * G::NT) == 0, "whole blocks and chunks");
    static_assert(G::LDS_ELEMS >= BM * BN, "the ring must hold one bfloat16 tile");
  }
  const bool full = m0 + BM <= a.M;  // no padding rows: no row mask
  // row mask of the last tile of a chunk: register group r4 of row block i holds rows
  // m0 + wm + 4 (lane / 32) + 32 i + 8 (r4 / 4) + q
  const int lim = a.M - m0 - wm - 4 * (lane >> 5);
  // Per token column j of this lane: the exponent offset, the sign of g, and the
  // target element this lane owns (tile row, or -1) with its value.
  // (ENT: cexp is -lse log2e, and a residual element p (wg + wx log2 p).)
  float cexp[NB], vt_val[NB], wg[NB], wx[NB];
  uint32_t sgn[NB];
  int trow[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int nl = n0 + wn + 32 * j + (lane & 31);  // token column within the chunk
    cexp[j] = -INFINITY;
    sgn[j] = 0u;
    trow[j] = -1;
    vt_val[j] = wg[j] = wx[j] = 0.f;
    if (nl < a.N) {
      const int64_t tg = tgv[j];
      if (ENT) {
        // (without an upstream gradient the entropy is not used: it may be NaN; and nor is lse without a loss)
        if (ev[j] != 0.f || tg != a.ignore_index) cexp[j] = -lsev[j] * kLog2e;
        if (ev[j] != 0.f) {
          wg[j] = -ev[j] * sv[j];
          wx[j] = -ev[j] * kLn2;
        }
      }
      if (tg != a.ignore_index) {
        float g = gv[j];
        if (tg < 0 || tg >= a.V) g = __builtin_nanf("");  // out of range: NaN row
        const float lse2 = lsev[j] * kLog2e;
        const float ag = __builtin_fabsf(g);
        if (!ENT) cexp[j] = __builtin_amdgcn_logf(ag) - lse2;  // log2|g| - lse log2e
        sgn[j] = !ENT && g < 0.f ? 0x80008000u : 0u;
        // the target element: inside the chunk (its padding rows stay zero), in this
        // wave's rows of the tile and in this lane half
        const int64_t rel = tg - a.gid0 - m0 - wm;
        if (tg - a.gid0 < a.M && rel >= 0 && rel < G::WM && (int)((rel >> 2) & 1) == (lane >> 5)) {
          trow[j] = (int)rel + wm;
          const float xt = __builtin_fmaf(ytv[j], kLog2e, -lse2), pt = __builtin_amdgcn_exp2f(xt);
          vt_val[j] = g * (pt - 1.f);
          if (ENT) vt_val[j] = __builtin_fmaf(pt, __builtin_fmaf(wx[j], fmaxf(xt, kLeastLog2), wg[j]), vt_val[j]);
        }
        if (ENT) wg[j] += g;
      }
    }
  }
  // G values of this lane, bfloat16 bits packed two per word: packed[j][i][r4/4]
  // holds vocabulary rows ml0 .. ml0 + 3 of token column nl.  Full tiles take the
  // loop without the padding-row mask.
  uint2 packed[NB][MB][4];
  auto residual = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int nl = n0 + wn + 32 * j + (lane & 31);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 16; r4 += 4) {
        // registers r4..r4+3 hold 4 consecutive vocabulary rows of token column nl
        const int ml0 = m0 + wm + 32 * i + acc_row(r4, lane);
        float v4[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float x = __builtin_fmaf(acc[i][j][r4 + q], kLog2e, cexp[j]);
          float e;
          if constexpr (ENT) {
            const float xl = fmaxf(x, kLeastLog2);
            e = __builtin_amdgcn_exp2f(xl) * __builtin_fmaf(wx[j], xl, wg[j]);
          } else {
            e = __builtin_amdgcn_exp2f(x);
          }
          v4[q] = (!MASKED || 32 * i + r4 / 4 * 8 + q < lim) ? e : 0.f;
        }
        if constexpr (kBlocked) {
          packed[j][i][r4 >> 2].x = E::pack2(v4[0], v4[1]) ^ sgn[j];
          packed[j][i][r4 >> 2].y = E::pack2(v4[2], v4[3]) ^ sgn[j];
        } else {
          const float sg = sgn[j] ? -1.f : 1.f;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v4[q] *= sg;
            Gs[(((uint32_t)nl / KB) * Vc + (uint32_t)(ml0 + q)) * KB + (uint32_t)nl % KB] = v4[q];
          }
          // 4 consecutive vocabulary rows: one 16-byte store into a 32-wide k-block
          *(float4*)(Gt + (((uint32_t)ml0 / KB) * Tc + (uint32_t)nl) * KB + (uint32_t)ml0 % KB) =
              make_float4(v4[0], v4[1], v4[2], v4[3]);
        }
      }
    if constexpr (!kBlocked) {
      if (trow[j] >= 0) {  // the target element, after this lane's own stores of it
        const uint32_t ml = (uint32_t)(m0 + trow[j]);
        Gs[(((uint32_t)nl / KB) * Vc + ml) * KB + (uint32_t)nl % KB] = vt_val[j];
        Gt[((ml / KB) * Tc + (uint32_t)nl) * KB + ml % KB] = vt_val[j];
      }
    }
  }
  };
  if (full)
    residual(std::false_type{});
  else
    residual(std::true_type{});
  if constexpr (kBlocked) {
    uint16_t* lds = (uint16_t*)smem;
    // G^T: the tile as rows of tokens, columns of vocabulary ids; a lane's 4
    // consecutive ids are one 8-byte write; then the target elements.
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r4 = 0; r4 < 16; r4 += 4) {
          const int tl = wn + 32 * j + (lane & 31), vl = wm + 32 * i + acc_row(r4, lane);
          *(uint2*)((char*)lds + tile_lds_byte<BN>(tl, vl)) = packed[j][i][r4 >> 2];
        }
    uint16_t tbits[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      tbits[j] = (uint16_t)(E::pack2(vt_val[j], 0.f) & 0xFFFFu);
      if (trow[j] >= 0)
        *(uint16_t*)((char*)lds + tile_lds_byte<BN>(wn + 32 * j + (lane & 31), trow[j])) = tbits[j];
    }
    __syncthreads();
    store_tile_blocked<G::NT, BN, BM>(lds, Gt, (uint32_t)m0 >> 6, Tc, (uint32_t)n0);
    __syncthreads();
    // G: the tile as rows of vocabulary ids, columns of tokens.
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r4 = 0; r4 < 16; r4 += 4) {
          const int tl = wn + 32 * j + (lane & 31), vl = wm + 32 * i + acc_row(r4, lane);
          const uint2 p = packed[j][i][r4 >> 2];
          char* base = (char*)lds;
          *(uint16_t*)(base + tile_lds_byte<BM>(vl, tl)) = (uint16_t)(p.x & 0xFFFFu);
          *(uint16_t*)(base + tile_lds_byte<BM>(vl + 1, tl)) = (uint16_t)(p.x >> 16);
          *(uint16_t*)(base + tile_lds_byte<BM>(vl + 2, tl)) = (uint16_t)(p.y & 0xFFFFu);
          *(uint16_t*)(base + tile_lds_byte<BM>(vl + 3, tl)) = (uint16_t)(p.y >> 16);
        }
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (trow[j] >= 0)
        *(uint16_t*)((char*)lds + tile_lds_byte<BM>(trow[j], wn + 32 * j + (lane & 31))) = tbits[j];
    __syncthreads();
    store_tile_blocked<G::NT, BM, BN>(lds, Gs, (uint32_t)n0 >> 6, Vc, (uint32_t)m0);
  }
}

// Column blocks of a dH / dW contraction, whose N is the hidden width d: BM-wide
// tiles of C^T rows (GM), except that a remainder of at most GW::BM - GM::BM
// columns joins the last full block, which then runs as one GW::BM-wide tile
// instead of leaving a block that is mostly padding (d = 2880: ten 256-wide
// blocks and one 320-wide block, not twelve 256-wide blocks of which the last
// holds 64 live columns).
struct ColBlocks {
  int n;      // column blocks
  bool wide;  // the last block is a GW tile
};
template <class GM, class GW>
__host__ __device__ inline ColBlocks col_blocks(int N) {
  static_assert(GW::BM >= GM::BM && GW::BN == GM::BN, "the wide tile only widens C^T rows");
  const int full = N / GM::BM, rem = N % GM::BM;
  if (GW::BM > GM::BM && full >= 1 && rem > 0 && rem <= GW::BM - GM::BM) return ColBlocks{full, true};
  return ColBlocks{(N + GM::BM - 1) / GM::BM, false};
}

// Stores a tile of sums: rows m0 .. of C, columns n0 .. n0 + BM - 1, added to what C
// holds if beta.
template <class G, bool RAGGED>
__device__ __forceinline__ void store_tile(const f32x16_t (&acc)[G::MB][G::NB], float* __restrict__ C,
                                           int64_t ldc, int M, int N, int m0, int n0, bool beta) {
  constexpr int MB = G::MB, NB = G::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = G::wave_m(wave), wn = G::wave_n(wave);
  // The epilogue takes a lane's row of C a batch of IB row blocks at a time: all
  // old values of the batch (beta = 1) are loaded before the first sum is stored,
  // so the lane waits for memory once per batch rather than once per 16-byte chunk
  // (a store to C ahead of the next load of C would keep the two in order).  Only
  // a RAGGED tile has columns at or past N.
  constexpr int IB = MB <= 4 ? MB : (MB + 1) / 2;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int m = m0 + wn + 32 * j + (lane & 31);
    if (m >= M) continue;
    float* crow = C + (int64_t)m * ldc;
#pragma unroll
    for (int i0 = 0; i0 < MB; i0 += IB) {
      float4 old[IB][4];
#pragma unroll
      for (int ii = 0; ii < IB; ++ii)
#pragma unroll
        for (int q = 0; q < 4; ++q) old[ii][q] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (beta) {
#pragma unroll
        for (int ii = 0; ii < IB; ++ii)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int i = i0 + ii;
            const int n = n0 + wm + 32 * i + acc_row(4 * q, lane);  // n .. n+3; N % 4 == 0
            if (i < MB && (!RAGGED || n < N)) old[ii][q] = *(const float4*)(crow + n);
          }
      }
#pragma unroll
      for (int ii = 0; ii < IB; ++ii)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int i = i0 + ii;
          const int n = n0 + wm + 32 * i + acc_row(4 * q, lane);
          if (i >= MB || (RAGGED && n >= N)) continue;
          const float4 c = old[ii][q];
          *(float4*)(crow + n) = make_float4(acc[i][j][4 * q] + c.x, acc[i][j][4 * q + 1] + c.y,
                                             acc[i][j][4 * q + 2] + c.z, acc[i][j][4 * q + 3] + c.w);
        }
    }
  }
}

// One dH or dW tile, rows m0 = mt * BN .. of C and columns n0 .. n0 + BM - 1, computed
// transposed, C^T[n][m] = sum_k A[n][k] B[m][k]: accumulator rows run along n, so each
// lane's group of 4 registers holds 4 consecutive columns of one row of C and the
// epilogue moves 16 bytes per access.  A is W or H read transposed (GC::ATR), or its
// k-blocked transposed copy.  A strip may hold several shards, and dH may be split into
// jobs along the vocabulary (see StageArgs): a dH tile runs the mainloop once per segment
// of its job, into the same accumulators.
// EDGE: the tile reaches past column d, which its stores leave out; SKIP: and so far that
// the waves skip the MFMAs of dead row blocks (RAGGED of the mainloop, whose branches
// cost more than they save where few blocks are dead).
template <class E, class GC, bool EDGE, bool SKIP>
__device__ __forceinline__ void contract_tile(const StageArgs& a, bool is_dh, int job, int mt, int n0,
                                              typename E::storage* smem) {
  using S = typename E::storage;
  constexpr int64_t KB = E::KB;
  const int64_t d = a.g.d, Tc = a.g.Tc;
  // contraction rows r0 .. r0 + rows - 1 of the strip (dH) or of the tokens (dW)
  // float32: two-level sums where the registers hold them; the 256-row tiles, whose do
  // not, add every segment to C by itself
  constexpr bool F32 = sizeof(S) == 4, TWO = F32 && GC::BM < 256;
  f32x16_t sum[TWO ? GC::MB : 1][GC::NB];
  if constexpr (TWO)
#pragma unroll
    for (int i = 0; i < GC::MB; ++i)
#pragma unroll
      for (int j = 0; j < GC::NB; ++j) sum[i][j] = f32x16_t{};
  auto mainloop = [&](f32x16_t(&acc)[GC::MB][GC::NB], const void* direct, const void* copy, int64_t r0,
                      int rows, const S* B, int64_t kblkb, int m0, int M) {
    if constexpr (GC::ATR) {
      GC::template run<SKIP>(acc, (const S*)direct, d, n0, (int)d, B, KB, m0, M, rows, smem, KB, kblkb,
                             TWO ? sum : nullptr);
      if constexpr (TWO) GC::flush(acc, sum);
    }
    else
      GC::template run<SKIP>(acc, (const S*)copy + r0 / KB * d * KB, KB, n0, (int)d, B, KB, m0, M,
                             (rows + (int)KB - 1) / (int)KB * (int)KB, smem, d * KB, kblkb);
  };
  f32x16_t acc[GC::MB][GC::NB];
#pragma unroll
  for (int i = 0; i < GC::MB; ++i)
#pragma unroll
    for (int j = 0; j < GC::NB; ++j) acc[i][j] = f32x16_t{};
  if (is_dh) {
    const StageJob jb = a.job[job];
    const int m0 = mt * GC::BN;
    for (int i = 0; i < jb.n_seg; ++i) {
      const StageSeg& sg = a.cseg[jb.seg + i];
      const int k0 = jb.n_seg == 1 ? jb.k0 : 0, rows = jb.n_seg == 1 ? jb.rows : sg.rows;
      mainloop(acc, (const S*)sg.w + (int64_t)k0 * d, a.Wt, sg.row0 + k0, rows,
               (const S*)a.Gt + (sg.row0 + k0) / KB * Tc * KB, Tc * KB, m0, a.c_N);
      if (F32 && !TWO && i + 1 < jb.n_seg) {
        store_tile<GC, EDGE>(acc, a.part + job * a.part_stride + a.c_t0 * d, d, a.c_N, (int)d, m0, n0,
                             i > 0 || jb.beta != 0);
#pragma unroll
        for (int x = 0; x < GC::MB; ++x)
#pragma unroll
          for (int y = 0; y < GC::NB; ++y) acc[x][y] = f32x16_t{};
      }
    }
    if constexpr (TWO) GC::flush(sum, acc);
    store_tile<GC, EDGE>(acc, a.part + job * a.part_stride + a.c_t0 * d, d, a.c_N, (int)d, m0, n0,
                         jb.beta != 0 || (F32 && !TWO && jb.n_seg > 1));
  } else {
    const int row = mt * GC::BN;
    int q = 0;
    while (q + 1 < a.n_cseg && row >= a.cseg[q + 1].row0) ++q;
    const StageSeg& sg = a.cseg[q];
    const int m0 = row - sg.row0;
    if (m0 >= sg.rows) return;  // padding of the segment
    mainloop(acc, (const S*)a.g.H + a.c_t0 * d, a.Ht, a.c_t0, a.c_N, (const S*)a.G + sg.row0 * KB,
             a.g.Vc * KB, m0, sg.rows);
    if constexpr (TWO) GC::flush(sum, acc);
    store_tile<GC, EDGE>(acc, sg.dw, d, sg.rows, (int)d, m0, n0, a.beta_w != 0);
  }
}

// One launch of the backward: the dH and dW tiles of one strip and the residual tiles of
// the next (which writes the other strip buffer).  XCD x runs cnt[p][x] tiles of the kind
// order[p], numbered from first[p][x], for p = 0, 1, 2: every XCD gets an even share of
// each kind, consecutive tiles of one kind stay on one XCD's L2, and the longest tiles go
// first so that the partly filled last round is made of the short ones.
template <class E, class GL, class GC, class GW, bool ENT>
__global__ void __launch_bounds__(GC::NT, GC::OCC* GC::NT / 256) bwd_stage_kernel(StageArgs a, StageSplit sp) {
  static_assert(GL::NT == GC::NT && GL::BN == GC::BN && GL::BM == GC::BM, "one tile shape");
  using S = typename E::storage;
  constexpr int LDS0 = GL::LDS_ELEMS > GC::LDS_ELEMS ? GL::LDS_ELEMS : GC::LDS_ELEMS;
  constexpr int LDS = LDS0 > GW::LDS_ELEMS ? LDS0 : GW::LDS_ELEMS;
  __shared__ __attribute__((aligned(16))) S smem[LDS];
  const int xcd = blockIdx.x % 8;
  int idx = blockIdx.x / 8, p = 0;
  while (p < 2 && idx >= sp.cnt[p][xcd]) idx -= sp.cnt[p++][xcd];
  idx += sp.first[p][xcd];
  const int kind = a.order[p];
  int mt, nt;
  if (kind == 2) {
    grouped_tile(idx, a.g.n_vt, (a.g.N + GL::BN - 1) / GL::BN, 4, mt, nt);
    const int row = mt * GL::BM;
    int q = 0;
    while (q + 1 < a.n_gseg && row >= a.gseg[q + 1].row0) ++q;
    GradArgs g = a.g;
    g.W = a.gseg[q].w;
    g.gid0 = a.gseg[q].gid0;
    g.M = a.gseg[q].rows;
    const int64_t row0 = a.gseg[q].row0;
    g.strip = (S*)g.strip + row0 * E::KB;
    g.strip_t = (S*)g.strip_t + row0 / E::KB * g.Tc * E::KB;
    grad_tile<E, GL, ENT>(g, a.entropy, a.grad_entropy, mt - (int)row0 / GL::BM, nt, smem);
    return;
  }
  const ColBlocks cb = col_blocks<GC, GW>(a.g.d);
  const int n_m = kind == 0 ? (a.c_N + GC::BN - 1) / GC::BN : a.w_tiles;
  const int per = n_m * cb.n, job = kind == 0 ? idx / per : 0;
  grouped_tile(idx - job * per, n_m, cb.n, 4, mt, nt);
  const int n0 = nt * GC::BM;
  const int cols = a.g.d - n0;  // live columns from n0 on
  if constexpr (GW::BM > GC::BM) {
    if (cb.wide && nt == cb.n - 1) {
      if (cols < GW::BM)
        contract_tile<E, GW, true, false>(a, kind == 0, job, mt, n0, smem);
      else
        contract_tile<E, GW, false, false>(a, kind == 0, job, mt, n0, smem);
      return;
    }
  }
  if (cols >= GC::BM)
    contract_tile<E, GC, false, false>(a, kind == 0, job, mt, n0, smem);
  else if (!GC::SKIPS || 2 * cols > GC::BM)
    contract_tile<E, GC, true, false>(a, kind == 0, job, mt, n0, smem);
  else if constexpr (GC::SKIPS)
    contract_tile<E, GC, true, true>(a, kind == 0, job, mt, n0, smem);
}

// Per-XCD split of n0 + n1 + n2 workgroups (workgroup b runs on XCD b % 8, so
// XCD x receives n/8 of them, one more for x < n%8): kinds 0 and 1 are spread
// as evenly as the capacity allows, kind 2 takes the rest.
static StageSplit split_stage(const int n_kind[3]) {
  StageSplit sp;
  const int n = n_kind[0] + n_kind[1] + n_kind[2];
  int cap[8];
  for (int x = 0; x < 8; ++x) cap[x] = n / 8 + (x < n % 8 ? 1 : 0);
  for (int t = 0; t < 2; ++t) {
    int give = n_kind[t];
    for (int x = 0; x < 8; ++x) {
      const int c = std::min(cap[x], n_kind[t] / 8);
      sp.cnt[t][x] = c;
      cap[x] -= c;
      give -= c;
    }
    for (int x = 0; give > 0; x = (x + 1) % 8)
      if (cap[x] > 0) {
        ++sp.cnt[t][x];
        --cap[x];
        --give;
      }
  }
  for (int x = 0; x < 8; ++x) sp.cnt[2][x] = cap[x];
  for (int t = 0; t < 3; ++t) {
    int f = 0;
    for (int x = 0; x < 8; ++x) {
      sp.first[t][x] = f;
      f += sp.cnt[t][x];
    }
  }
  return sp;
}

template <class E, bool ENT, class GL, class GC, class GW = GC>
static bool launch_stage_g(const StageArgs& a, hipStream_t s) {
  const int n_tb = (a.g.N + GL::BN - 1) / GL::BN, n_cb = (a.c_N + GC::BN - 1) / GC::BN;
  const int n_nb = col_blocks<GC, GW>(a.g.d).n;
  const int tiles[3] = {a.n_job * n_cb * n_nb, a.w_tiles * n_nb, a.g.n_vt * n_tb};
  int n_kind[3], n = 0;
  for (int p = 0; p < 3; ++p) n += n_kind[p] = tiles[a.order[p]];
  if (n == 0) return true;
  hipLaunchKernelGGL((bwd_stage_kernel<E, GL, GC, GW, ENT>), dim3((unsigned)n), dim3(GC::NT), 0, s, a,
                     split_stage(n_kind));
  return launched_ok();
}
template <class E, bool ENT>
static bool launch_stage(int cls, const StageArgs& a, hipStream_t s) {
  using C = Cfg<E>;
  if (cls == 1) return launch_stage_g<E, ENT, typename C::Res128x64, typename C::Tr128x64>(a, s);
  if (cls == 2) return launch_stage_g<E, ENT, typename C::Res128, typename C::Tr128>(a, s);
  const bool whole = a.g.d % E::KB == 0;
  if constexpr (sizeof(typename E::storage) == 2) {
    if (cls == 0 && whole) return launch_stage_g<E, ENT, typename C::Logits, typename C::Tr256, typename C::Tr320>(a, s);
    if (cls == 0) return launch_stage_g<E, ENT, typename C::LogitsTail, typename C::Tr256, typename C::Tr320>(a, s);
  }
  if (cls != 3) return false;
  if (whole) return launch_stage_g<E, ENT, typename C::Logits, typename C::Mm, typename C::MmWide>(a, s);
  return launch_stage_g<E, ENT, typename C::LogitsTail, typename C::Mm, typename C::MmWide>(a, s);
}

}  // namespace vpce
