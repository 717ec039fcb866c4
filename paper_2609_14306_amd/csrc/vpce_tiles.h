// Tiles of the products of the vocabulary projection: element types, mainloops, the online
// softmax fold of a tile, and which tile a workgroup runs.  vpce_kernels.hip says how they are put
// together; its kernels, those of the backward (vpce_backward.h) and those of the scoring calls
// (vpce_score.hip) are built on these.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "vpce_internal.h"

namespace vpce {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------------------
// Element policies.  VEC: elements per 16 bytes.
// KB: elements of one 128-byte k-block of the k-blocked backward workspaces (and of
// one row of a direct-to-LDS slice).  frag16 / mma16: one 16-byte operand fragment
// per lane (8 bfloat16 or 4 float32 k values) and the MFMA work it feeds.
struct Bf16 {
  using storage = uint16_t;
  using frag16 = bf16x8_t;
  static constexpr int VEC = 8, KB = 64;
  __device__ static f32x16_t mma16(frag16 a, frag16 b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // Two float32 values rounded to nearest even, packed low then high (one
  // v_cvt_pk_bf16_f32).
  __device__ static uint32_t pack2(float lo, float hi) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
  }
};
typedef float f32x4_t __attribute__((ext_vector_type(4)));
struct F32 {
  using storage = float;
  using frag16 = f32x4_t;
  static constexpr int VEC = 4, KB = 32;
  // Lane half h holds k = 4h .. 4h + 3 of an 8-wide k group in both operands; MFMA q
  // takes element q, i.e. k = q (lanes 0-31) and 4 + q (lanes 32-63): the four MFMAs
  // together cover the group (the contraction order within it is a permutation).
  __device__ static f32x16_t mma16(frag16 a, frag16 b, f32x16_t c) {
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[0], b[0], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[1], b[1], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[2], b[2], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a[3], b[3], c, 0, 0, 0);
  }
};

// Accumulator layout of a 32x32 MFMA block: lane l, register r holds
// row 8*(r/4) + 4*(l/32) + r%4 and column l%32.
__device__ __forceinline__ int acc_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// ---------------------------------------------------------------------------
// Tile GEMM fed by direct global -> LDS loads (global_load_lds_dwordx4, 16 bytes
// per lane straight into LDS, no staging registers) through a ring of two
// k-slices of 128-byte rows: 64 bfloat16 or 32 float32 k values per row.  A
// 16-byte fragment feeds one 32x32x16 bf16 MFMA or four 32x32x2 f32 MFMAs (see
// the element policies); everything else is the same for both types.
//
// LDS slice layout: the A rows then the B rows, 128 bytes (eight 16-byte
// chunks) per row, chunk c of row r stored in slot c ^ ((r >> 1) & 7): the 16
// lanes of one LDS read phase (16 consecutive rows, same chunk) hit 16 distinct
// 4-bank groups, and each load instruction writes 1 KiB contiguously (8 rows).
//
// Schedule of one wave (slice kt lives in ring slot kt & 1; sub-step kk covers
// k = 16 kk .. 16 kk + 15 of the slice):
//   sub-steps 0..2: issue the MFMAs of sub-step kk, each followed by one LDS read
//                   of a fragment of sub-step kk+1 into the spare register set;
//   sub-step 3:     wait for this wave's loads of slice kt+1, barrier, then the
//                   MFMAs of sub-step 3 interleaved with the reads of slice kt+1
//                   sub-step 0.
// The loads of slice kt+2 go out one per two MFMAs, half during sub-step 3 of
// slice kt (into slot kt & 1: every wave finished reading slice kt before the
// barrier) and half during sub-step 0 of slice kt+1.  The MFMAs never wait on an
// LDS read issued in the same sub-step, the only barrier of a slice sits where
// every wave holds a sub-step of fragments in registers, each slice's loads have
// three or four sub-steps of MFMAs to land, and no burst of memory instructions
// ever stands in front of a wave's next MFMA.
// The loads are issued from inline assembly with a scalar base (the tile's
// first row at the slice's k offset) and a 32-bit per-lane byte offset, so that
// the compiler neither drains the loads before each LDS read (it cannot tell
// which ring slot a read touches) nor keeps 64-bit addresses per load.
// Completion is tracked by hand with vmcnt: loads return in issue order and the
// only loads a wave has in flight are its slice loads.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  // s_waitcnt simm16 on gfx9: vmcnt[3:0] | expcnt[6:4] | lgkmcnt[11:8] | vmcnt[5:4] << 14
  __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}
__device__ __forceinline__ void wait_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// One direct-to-LDS load from a scalar base.  The hazards the compiler's hazard
// recognizer cannot see inside inline assembly are covered here: five wait states
// before the load in case a VALU instruction (v_readlane of a spilled value, a
// carry-out) wrote the base SGPRs just before it, and one after the M0 write,
// which an LDS DMA reads.
__device__ __forceinline__ void lds_dma16x1(const void* sbase, uint32_t o0, uint32_t l0) {
  uint32_t m0v = l0;
  asm volatile("s_nop 4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               : "+{m0}"(m0v)
               : "v"(o0), "s"(sbase)
               : "memory");
}

// The same load from 64-bit per-lane addresses, for the last slice of a contraction
// whose K is no multiple of the slice depth: the lanes whose 16-byte chunk lies past K
// read zeros from zero_chunk instead (a product with another row's values would not
// be harmless: they may be infinite or NaN).
static __device__ uint4 zero_chunk = {0u, 0u, 0u, 0u};
__device__ __forceinline__ void lds_dma16_lane(const void* addr, uint32_t l0) {
  uint32_t m0v = l0;
  asm volatile("s_nop 4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               : "+{m0}"(m0v)
               : "v"(addr)
               : "memory");
}

// An operand whose contraction index is its row index, read transposed from LDS: a
// slice is E::KB rows (k) of COLS values (n, the tile's rows of C^T), copied row by row
// by the direct-to-LDS loads.  bfloat16 fragments come from gfx950's LDS transpose read
// (ds_read_b64_tr_b16: in each group of 16 lanes, lane a supplies the four values at its
// address, and lane i receives value i % 4 of lanes i / 4, 4 + i / 4, 8 + i / 4 and
// 12 + i / 4, i.e. a 4 x 16 block transposed), two per 8-value fragment; float32 ones
// from four 4-byte reads.  The 16-byte chunks of k-row r are swizzled by swz(r) so that
// the rows that one read touches lie in different banks.
typedef short s16x4_t __attribute__((ext_vector_type(4)));
template <class E, int COLS, int NWAVES>
struct TrOperand {
  using S = typename E::storage;
  using F16 = typename E::frag16;
  static constexpr int ROW_BYTES = COLS * (int)sizeof(S);
  static constexpr int CPR = ROW_BYTES / 16;  // chunks per k-row
  static_assert(ROW_BYTES % 128 == 0 && ROW_BYTES >= 256, "the swizzle needs two or four bank groups");
  // Bank group (64 bytes) of k-row r's chunk 0 is r ROW_BYTES / 64 mod 4: 0 for every row
  // where ROW_BYTES is a multiple of 256, alternating with r otherwise (640).
  __device__ __forceinline__ static int swz(int k) {
    if (sizeof(S) == 4) return 8 * ((k >> 2) & 1);
    return ROW_BYTES % 256 == 0 ? 4 * (k & 3) : 4 * ((k >> 1) & 1);
  }
  // Chunk (wave + q NWAVES) * 64 + lane of the slice, row by row, is what this lane loads
  // with load q: its k-row and its place in the row.
  __device__ __forceinline__ static int place(int q, int wave, int lane) {
    return (wave + q * NWAVES) * 64 + lane;
  }
  // Byte offset, from the slice's first row, of the chunk that this lane loads with
  // load q: k-row min(row, last), column chunk clamped to the last one below `cols`
  // (columns past it feed rows of C^T that are never stored; k-rows past `last` meet
  // zeros of the other operand).
  __device__ __forceinline__ static uint32_t offset(int q, int wave, int lane, int64_t ld, int cols,
                                                    int last) {
    const int u = place(q, wave, lane), r = u / CPR, c = (u % CPR) ^ swz(r);
    return (uint32_t)(min(r, last) * ld * (int64_t)sizeof(S)) + 16u * (uint32_t)min(c, cols / E::VEC - 1);
  }
  // Lane's byte offset of the fragment of 32-wide block n0 at sub-step 0, and the read.
  __device__ __forceinline__ static uint32_t frag_offset(int n0, int lane) {
    if constexpr (sizeof(S) == 2) {
      const int k = 8 * (lane >> 5) + ((lane & 15) >> 2);
      const int n = n0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      return (uint32_t)(k * ROW_BYTES + (((n >> 3) ^ swz(k)) << 4) + (n & 7) * 2);
    } else {
      const int k = 4 * (lane >> 5), n = n0 + (lane & 31);
      return (uint32_t)(k * ROW_BYTES + (((n >> 2) ^ swz(k)) << 4) + (n & 3) * 4);
    }
  }
  __device__ __forceinline__ static F16 frag(const char* p, int kk) {
    if constexpr (sizeof(S) == 2) {
      using P = __attribute__((address_space(3))) s16x4_t*;
      typedef short s16x8_t __attribute__((ext_vector_type(8)));
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + kk * 16 * ROW_BYTES));
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + (kk * 16 + 4) * ROW_BYTES));
      return __builtin_bit_cast(F16, (s16x8_t)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      F16 f;
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = *(const float*)(p + (kk * 8 + e) * ROW_BYTES);
      return f;
    }
  }
};

// KTAIL_: K may be any number of whole 16-byte chunks; otherwise it is a multiple of
// the slice depth.
// ATR_: A is [K][lda] with its rows along the contraction, read transposed (TrOperand);
// K is its number of rows, any number, and B is whole slices that hold zeros past K.
// run() with a `sum`: the accumulators are added to it and cleared every kFlush slices,
// and left with what has gathered since (float32: a chain of 1024 products rounds less
// than one of 25000, whose error shows in dH).
constexpr int kFlush = 32;
template <int BM_, int BN_, int WGM_, int WGN_, class E = Bf16, bool KTAIL_ = false, bool ATR_ = false>
struct GemmDma {
  using S = typename E::storage;
  using F16 = typename E::frag16;
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_;
  static constexpr int NT = 64 * WGM * WGN, NWAVES = WGM * WGN;
  // Two wavefronts per SIMD with 256 registers each: one 512-thread workgroup per CU
  // (whose ring takes 128 to 160 KiB of LDS) or two 256-thread ones.
  static constexpr int OCC = NT == 512 ? 1 : 2;
  static constexpr int WM = BM / WGM, WN = BN / WGN, MB = WM / 32, NB = WN / 32;
  static_assert(WM % 32 == 0 && WN % 32 == 0, "wave tile must be whole 32x32 blocks");
  static constexpr int STAGES = 2;        // ring slots
  static constexpr int ROW_BYTES = 128;
  static constexpr int BK = E::KB;        // k values per slice: one k-block of the layout
  static constexpr bool KTAIL = KTAIL_, ATR = ATR_;
  static constexpr bool SKIPS = true;             // run<true> skips dead row blocks
  static constexpr int NKK = ROW_BYTES / 32;      // sub-steps per slice (two 16-byte chunks each)
  static constexpr int CPR = ROW_BYTES / 16;      // 16-byte chunks per row
  static constexpr int RPW = 256 / ROW_BYTES;     // rows per 64-bank (256-byte) window
  static constexpr int RPI = 1024 / ROW_BYTES;    // rows per 1 KiB load instruction
  static constexpr int SLICE_BYTES = (BM + BN) * ROW_BYTES;
  static constexpr int A_LOADS = BM / RPI / NWAVES;  // load instructions per wave and slice
  static constexpr int B_LOADS = BN / RPI / NWAVES;
  static_assert(BM % (RPI * NWAVES) == 0 && BN % (RPI * NWAVES) == 0, "whole load groups per wave");
  using TrA = TrOperand<E, BM, NWAVES>;
  static constexpr int NLOADS = A_LOADS + B_LOADS;  // per wave and slice
  // the loads of a slice go out in two halves, the larger first
  static constexpr int HALF0 = (NLOADS + 1) / 2, HALF1 = NLOADS - HALF0;
  static constexpr int NM = MB * NB, NR = MB + NB;   // MFMAs and fragment reads per sub-step
  // one load per LSTEP MFMAs of a sub-step
  static constexpr int LSTEP = 2 * HALF0 <= NM + 1 ? 2 : 1;
  static_assert(NR <= NM && LSTEP * (HALF0 - 1) < NM, "interleave slots");
  static constexpr int LDS_ELEMS = STAGES * SLICE_BYTES / (int)sizeof(S);
  static_assert(STAGES * SLICE_BYTES <= 160 * 1024, "LDS");

  // Chunk c of slice row r lives in slot c ^ key(r): within one 256-byte window
  // the rows sit at distinct offsets, and key(r) differs for the CPR rows that
  // share a window offset, so a read phase of 16 consecutive rows at one chunk
  // touches 16 distinct 4-bank groups.
  __device__ __forceinline__ static int key(int r) { return (r / RPW) % CPR; }

  __device__ __forceinline__ static int wave_m(int wave) { return (wave / WGN) * WM; }
  __device__ __forceinline__ static int wave_n(int wave) { return (wave % WGN) * WN; }

  __device__ __forceinline__ static uint32_t slot_bytes(int kt) {
    return (uint32_t)((kt % STAGES) * SLICE_BYTES);
  }

  // Load instruction q of a wave covers the RPI slice rows starting at
  // (wave + q * NWAVES) * RPI; A rows come first.  Rows at or beyond M (N) are
  // clamped to the last row: they only feed accumulator rows (columns) that are
  // never stored.
  struct Loads {
    const char* baseA;  // byte address of the tile's first A row (k = 0)
    const char* baseB;
    int64_t kblkA, kblkB;  // elements between consecutive k-blocks (E::KB wide)
    // KTAIL: the slice that reaches past K and its live chunks; ATR: that slice and its
    // live rows, A's row pitch and live columns
    int tail_kt, tail_chunks, tail_rows, colsA;
    int64_t ldA;
    uint32_t offA[A_LOADS], offB[B_LOADS];  // per-lane byte offsets from the bases
  };

  __device__ __forceinline__ static void plan(Loads& L, const S* __restrict__ A, int64_t lda,
                                              int m0, int M, const S* __restrict__ B, int64_t ldb,
                                              int n0, int N, int wave, int lane) {
    const int ma = min(m0, M - 1), nb = min(n0, N - 1);
    if constexpr (ATR)
      L.baseA = (const char*)(A + m0);
    else
      L.baseA = (const char*)(A + (int64_t)ma * lda);
    L.baseB = (const char*)(B + (int64_t)nb * ldb);
    const int row_in = lane / CPR;
#pragma unroll
    for (int q = 0; q < A_LOADS; ++q) {
      if constexpr (ATR) {
        L.offA[q] = TrA::offset(q, wave, lane, lda, M - m0, BK - 1);
        continue;
      }
      const int r = (wave + q * NWAVES) * RPI + row_in;
      const int c = (lane % CPR) ^ key(r);
      L.offA[q] = (uint32_t)((min(m0 + r, M - 1) - ma) * lda * (int64_t)sizeof(S)) + 16u * c;
    }
#pragma unroll
    for (int q = 0; q < B_LOADS; ++q) {
      const int r = (wave + (A_LOADS + q) * NWAVES) * RPI + row_in;  // >= BM
      const int c = (lane % CPR) ^ key(r);
      L.offB[q] = (uint32_t)((min(n0 + r - BM, N - 1) - nb) * ldb * (int64_t)sizeof(S)) + 16u * c;
    }
  }

  // Load q (operand A's loads, then B's) of slice kt, into ring slot kt % STAGES:
  // it fills the 1 KiB at (wave + q * NWAVES) KiB of the slot.
  __device__ __forceinline__ static void issue_one(const Loads& L, int kt, int q, uint32_t lds0,
                                                   int wave) {
    constexpr int KB = E::KB;
    const int64_t k0 = (int64_t)kt * BK;
    const uint32_t l = lds0 + slot_bytes(kt) + (uint32_t)(wave * 1024) + q * NWAVES * 1024;
    if constexpr (KTAIL) {
      if (kt == L.tail_kt) {
        const int lane = threadIdx.x & 63;
        const int c = (lane % CPR) ^ key((wave + q * NWAVES) * RPI + lane / CPR);
        const char* p = q < A_LOADS
                            ? L.baseA + (k0 / KB) * L.kblkA * (int64_t)sizeof(S) + L.offA[q < A_LOADS ? q : 0]
                            : L.baseB + (k0 / KB) * L.kblkB * (int64_t)sizeof(S) + L.offB[q < A_LOADS ? 0 : q - A_LOADS];
        lds_dma16_lane(c < L.tail_chunks ? (const void*)p : (const void*)&zero_chunk, l);
        return;
      }
    }
    if constexpr (ATR) {
      if (q < A_LOADS && kt == L.tail_kt) {
        const uint32_t o = TrA::offset(q, wave, (int)(threadIdx.x & 63), L.ldA, L.colsA, L.tail_rows - 1);
        lds_dma16_lane(L.baseA + (k0 / KB) * L.kblkA * (int64_t)sizeof(S) + o, l);
        return;
      }
    }
    if (q < A_LOADS)
      lds_dma16x1(L.baseA + ((k0 / KB) * L.kblkA + (k0 % KB)) * (int64_t)sizeof(S), L.offA[q], l);
    else
      lds_dma16x1(L.baseB + ((k0 / KB) * L.kblkB + (k0 % KB)) * (int64_t)sizeof(S), L.offB[q - A_LOADS], l);
  }

  // Fragment idx (the MB A blocks, then the NB B blocks) of sub-step kk at slot
  // byte address `slot`: lane l takes row l % 32 of the block and the 16 bytes of
  // chunk 2 kk + l / 32 (bf16: k = 16 kk + 8 (l / 32) + 0..7).
  __device__ __forceinline__ static F16 read_one(const char* slot, int wm, int wn, int kk, int lane,
                                                 int idx) {
    const int chunk = 2 * kk + (lane >> 5);
    const int row = idx < MB ? wm + 32 * idx + (lane & 31) : BM + wn + 32 * (idx - MB) + (lane & 31);
    return *(const F16*)(slot + row * ROW_BYTES + ((chunk ^ key(row)) << 4));
  }

  // Wait until at most n slices' loads (0 or 1) of this wave are in flight; loads return
  // in issue order.
  __device__ __forceinline__ static void wait_slices(int n) {
    if (n <= 0)
      wait_vmcnt<0>();
    else
      wait_vmcnt<NLOADS>();
  }

  // sum += acc, acc = 0
  __device__ __forceinline__ static void flush(f32x16_t (&acc)[MB][NB], f32x16_t (*sum)[NB]) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        sum[i][j] += acc[i][j];
        acc[i][j] = f32x16_t{};
      }
  }

  // acc += A[m0 : m0+BM, 0:K] B[n0 : n0+BN, 0:K]^T; requires m0 < M and n0 < N.
  // Element (r, k) of A is at A[(k / KB) kblka + r lda + k % KB] with KB = E::KB
  // (row-major: kblka = KB; k-blocked: lda = KB, kblka = rows * KB), likewise for B.
  // RAGGED: the tile reaches past row M of A; each wave skips the MFMAs (and the
  // fragment reads) of its 32-row blocks of A that lie wholly at or past M, whose
  // accumulators stay zero and are never stored.
  // LDS is free again for the caller when run() returns.
  template <bool RAGGED = false>
  __device__ __forceinline__ static void run(f32x16_t (&acc)[MB][NB], const S* __restrict__ A,
                                             int64_t lda, int m0, int M, const S* __restrict__ B,
                                             int64_t ldb, int n0, int N, int K, S* smem,
                                             int64_t kblka = E::KB, int64_t kblkb = E::KB,
                                             f32x16_t (*sum)[NB] = nullptr) {
    // The wave index is made scalar so that every branch on it is a scalar branch.
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave_m(wave), wn = wave_n(wave);
    const int nk = KTAIL || ATR ? (K + BK - 1) / BK : K / BK;
    if (nk <= 0) return;
    // row blocks of A with live rows (wave-uniform); MB unless RAGGED
    const int mb_live = RAGGED ? max(0, min(MB, (M - m0 - wm + 31) / 32)) : MB;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) S*)smem;
    Loads L;
    plan(L, A, lda, m0, M, B, ldb, n0, N, wave, lane);
    L.kblkA = kblka;
    L.kblkB = kblkb;
    if constexpr (KTAIL) {
      L.tail_kt = K % BK ? nk - 1 : -1;
      L.tail_chunks = K % BK / E::VEC;
    }
    uint32_t fragA[MB];  // ATR: this lane's offsets of its A fragments
    if constexpr (ATR) {
      L.tail_kt = K % BK ? nk - 1 : -1;
      L.tail_rows = K % BK;
      L.kblkA = BK * lda;
      L.ldA = lda;
      L.colsA = M - m0;
#pragma unroll
      for (int i = 0; i < MB; ++i) fragA[i] = TrA::frag_offset(wm + 32 * i, lane);
    }
    auto read_a = [&](const char* slot, int kk, int i) -> F16 {
      if constexpr (ATR)
        return TrA::frag(slot + fragA[i], kk);
      else
        return read_one(slot, wm, wn, kk, lane, i);
    };
    // prologue: the first min(STAGES, nk) slices, whole; wait for slice 0
    const int pro = min(STAGES, nk);
    for (int kt = 0; kt < pro; ++kt)
#pragma unroll
      for (int q = 0; q < NLOADS; ++q) issue_one(L, kt, q, lds0, wave);
    wait_slices(pro - 1);
    __builtin_amdgcn_s_barrier();
    const char* ring = (const char*)smem;
    // A fragments are single-buffered: each is re-read for the next sub-step right
    // after its last MFMA of this one.  B fragments are double-buffered and read
    // during the first MFMAs of the sub-step.  The MFMAs go in snake order (row
    // block i takes its column blocks forwards for even i, backwards for odd i), so
    // that consecutive MFMAs share an operand.
    F16 a[MB], b[2][NB];
#pragma unroll
    for (int idx = 0; idx < NR; ++idx) {
      if (idx < MB)
        a[idx] = read_a(ring, 0, idx);
      else
        b[0][idx - MB] = read_one(ring, wm, wn, 0, lane, idx);
    }
    for (int kt = 0; kt < nk; ++kt) {
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        const int cur = kk & 1;
        // where the fragments of the next sub-step come from
        const char* src;
        int skk;
        if (kk + 1 < NKK) {
          src = ring + slot_bytes(kt);
          skk = kk + 1;
        } else {
          // Slice kt+1 must have landed; no other load is in flight.  Taken on the last
          // slice too (one spare barrier, fragments read from an idle slot and never
          // used): no branch around the LDS reads, so the compiler's count of reads in
          // flight stays exact.
          wait_vmcnt<0>();
          wait_lgkmcnt0();  // this wave's reads of slice kt
          __builtin_amdgcn_s_barrier();
          src = ring + slot_bytes(kt + 1);
          skk = 0;
        }
        // The loads of slice kt+STAGES go out in two halves: the first during the
        // last sub-step of slice kt (after the barrier: every wave has finished
        // reading slice kt, whose slot they refill), the second during the first
        // sub-step of slice kt+1 (the prologue issued the first STAGES slices).
        const int dq0 = kk == NKK - 1 ? 0 : HALF0;
        const int dn = kk == NKK - 1 ? HALF0 : HALF1;
        const int dslice = kk == NKK - 1 ? kt + STAGES : kt + STAGES - 1;
        const bool dvalid = (kk == NKK - 1 || (kk == 0 && kt >= 1)) && dslice < nk;
        __builtin_amdgcn_sched_barrier(0);
        // One MFMA, then the fragment reads it frees for the next sub-step, then
        // (every other MFMA) one load: the wave never holds a burst of memory
        // instructions in front of its next MFMA.
#pragma unroll
        for (int idx = 0; idx < NM; ++idx) {
          const int i = idx / NB, jj = idx % NB, j = (i & 1) ? NB - 1 - jj : jj;
          const bool live = !RAGGED || i < mb_live;
          if (live) acc[i][j] = E::mma16(a[i], b[cur][j], acc[i][j]);
          __builtin_amdgcn_sched_barrier(0);
          if (idx < NB) b[cur ^ 1][idx] = read_one(src, wm, wn, skk, lane, MB + idx);
          if (jj == NB - 1 && live) a[i] = read_a(src, skk, i);
          if (idx % LSTEP == 0 && idx / LSTEP < dn && (kk == NKK - 1 || kk == 0) && dvalid)
            issue_one(L, dslice, dq0 + idx / LSTEP, lds0, wave);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (sum != nullptr && kt % kFlush == kFlush - 1) flush(acc, sum);
    }
    // no wave may still be reading the ring, nor a load writing it, when the caller
    // reuses LDS
    wait_vmcnt<0>();
    wait_lgkmcnt0();
    __builtin_amdgcn_s_barrier();
  }
};

// ---------------------------------------------------------------------------
// Small tiles for problems whose 256 x 256 tiles would leave most of the chip idle or
// be mostly padding: the same slices, swizzle and direct-to-LDS loads, but a ring of
// STAGES slices of which all but one are in flight, and one plain loop over slices
// (wait, barrier, refill, multiply).  What bounds these problems is the stream of W
// from memory: a CU keeps (STAGES - 1) slices of it in flight, and the ring runs on
// across tile boundaries (stream_fwd_kernel), so that no tile starts on an empty pipe.
// Forward of T = 40, d = 4096, V = 151936 in bfloat16: 1549 us with 32 workgroups of
// 256 x 256 tiles, 310 with 256 of them, 234 with these (5.3 TB/s of W).
// ATR_: A is read transposed, as in GemmDma.
template <int BM_, int BN_, int WGM_, int WGN_, int STAGES_, class E, bool ATR_ = false>
struct Ring {
  using S = typename E::storage;
  using F16 = typename E::frag16;
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, STAGES = STAGES_;
  static constexpr int NT = 64 * WGM * WGN, NWAVES = WGM * WGN;
  static constexpr int WM = BM / WGM, WN = BN / WGN, MB = WM / 32, NB = WN / 32;
  static_assert(WM % 32 == 0 && WN % 32 == 0, "wave tile must be whole 32x32 blocks");
  static constexpr int BK = E::KB, CPR = 8;  // 128-byte slice rows of eight 16-byte chunks
  static constexpr int SLICE_BYTES = (BM + BN) * 128;
  static constexpr int LDS_BYTES = STAGES * SLICE_BYTES;
  static constexpr int OCC = LDS_BYTES <= 80 * 1024 ? 2 : 1;  // workgroups per CU
  static constexpr int A_LOADS = BM / 8 / NWAVES, B_LOADS = BN / 8 / NWAVES;
  static_assert(BM % (8 * NWAVES) == 0 && BN % (8 * NWAVES) == 0, "whole load groups per wave");
  static constexpr int NLOADS = A_LOADS + B_LOADS;
  static constexpr bool ATR = ATR_, SKIPS = false;
  static constexpr int LDS_ELEMS = LDS_BYTES / (int)sizeof(S);
  using TrA = TrOperand<E, BM, NWAVES>;
  static_assert(STAGES >= 3 && (STAGES - 2) * NLOADS < 64 && LDS_BYTES <= 160 * 1024, "ring");
  static_assert(2 * WGM * BN * 4 <= LDS_BYTES, "write_partials' exchange");

  __device__ __forceinline__ static int wave_m(int wave) { return (wave / WGN) * WM; }
  __device__ __forceinline__ static int wave_n(int wave) { return (wave % WGN) * WN; }
  __device__ __forceinline__ static int key(int r) { return (r >> 1) & 7; }

  // Per-lane byte offsets of an operand's loads: load q of a wave covers the eight rows
  // from (wave + q * NWAVES) * 8; rows at or past `rows` repeat the last one.
  template <int N>
  __device__ __forceinline__ static void offsets(uint32_t (&off)[N], int rows, int64_t ld, int wave,
                                                 int lane) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int r = (wave + q * NWAVES) * 8 + lane / 8;
      off[q] = (uint32_t)(min(r, rows - 1) * ld * (int64_t)sizeof(S)) + 16u * ((lane & 7) ^ key(r));
    }
  }
  // The loads of one operand's part of a slice into LDS at l0.  chunks: live 16-byte
  // chunks of the slice's rows (8, or fewer where the slice reaches past K: those read
  // zeros).
  template <int N>
  __device__ __forceinline__ static void issue(const char* base, const uint32_t (&off)[N],
                                               int chunks, uint32_t l0, int wave, int lane) {
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const uint32_t l = l0 + (uint32_t)(wave + q * NWAVES) * 1024u;
      if (chunks == CPR) {
        lds_dma16x1(base, off[q], l);
      } else {
        const int c = (lane & 7) ^ key((wave + q * NWAVES) * 8 + lane / 8);
        lds_dma16_lane(c < chunks ? (const void*)(base + off[q]) : (const void*)&zero_chunk, l);
      }
    }
  }
  // acc += the product of one slice at LDS address `slot` (A rows, then B rows).
  __device__ __forceinline__ static void multiply(f32x16_t (&acc)[MB][NB], const char* slot, int wm,
                                                  int wn, int lane) {
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int chunk = 2 * kk + (lane >> 5);
      F16 fa[MB], fb[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const int r = wm + 32 * i + (lane & 31);
        if constexpr (ATR)
          fa[i] = TrA::frag(slot + TrA::frag_offset(wm + 32 * i, lane), kk);
        else
          fa[i] = *(const F16*)(slot + r * 128 + ((chunk ^ key(r)) << 4));
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int r = wn + 32 * j + (lane & 31);
        fb[j] = *(const F16*)(slot + (BM + r) * 128 + ((chunk ^ key(r)) << 4));
      }
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = E::mma16(fa[i], fb[j], acc[i][j]);
    }
  }

  // sum += acc, acc = 0
  __device__ __forceinline__ static void flush(f32x16_t (&acc)[MB][NB], f32x16_t (*sum)[NB]) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        sum[i][j] += acc[i][j];
        acc[i][j] = f32x16_t{};
      }
  }

  // One tile of its own (the interface of GemmDma::run): acc += A B^T.  A part slice at
  // the end reads zeros past K, or, with ATR, repeats A's last row against B's zeros.
  template <bool RAGGED = false>
  __device__ __forceinline__ static void run(f32x16_t (&acc)[MB][NB], const S* __restrict__ A,
                                             int64_t lda, int m0, int M, const S* __restrict__ B,
                                             int64_t ldb, int n0, int N, int K, S* smem,
                                             int64_t kblka = E::KB, int64_t kblkb = E::KB,
                                             f32x16_t (*sum)[NB] = nullptr) {
    static_assert(!RAGGED, "one row block per wave: nothing to skip");
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave_m(wave), wn = wave_n(wave);
    const int nk = (K + BK - 1) / BK, tail = K % BK;
    if (nk <= 0) return;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) S*)smem;
    const char* baseA = (const char*)(ATR ? A + m0 : A + (int64_t)m0 * lda);
    const char* baseB = (const char*)(B + (int64_t)n0 * ldb);
    const int64_t stepA = (ATR ? BK * lda : kblka) * (int64_t)sizeof(S);
    const int64_t stepB = kblkb * (int64_t)sizeof(S);
    uint32_t offA[A_LOADS], offB[B_LOADS];
    if constexpr (ATR) {
#pragma unroll
      for (int q = 0; q < A_LOADS; ++q) offA[q] = TrA::offset(q, wave, lane, lda, M - m0, BK - 1);
    } else {
      offsets(offA, M - m0, lda, wave, lane);
    }
    offsets(offB, N - n0, ldb, wave, lane);
    int loaded = 0, l_slot = 0, slot = 0;
    auto load_next = [&]() {
      const uint32_t l = lds0 + (uint32_t)(l_slot * SLICE_BYTES);
      const bool part = tail != 0 && loaded == nk - 1;
      if (ATR && part) {
#pragma unroll
        for (int q = 0; q < A_LOADS; ++q)
          lds_dma16_lane(baseA + TrA::offset(q, wave, lane, lda, M - m0, tail - 1),
                         l + (uint32_t)(wave + q * NWAVES) * 1024u);
      } else {
        issue(baseA, offA, part ? tail / E::VEC : CPR, l, wave, lane);
      }
      issue(baseB, offB, part && !ATR ? tail / E::VEC : CPR, l + BM * 128, wave, lane);
      baseA += stepA;
      baseB += stepB;
      l_slot = l_slot + 1 == STAGES ? 0 : l_slot + 1;
      ++loaded;
    };
    for (int k = 0; k < min(STAGES - 1, nk); ++k) load_next();
    for (int it = 0; it < nk; ++it) {  // (the waits of stream_fwd_kernel)
      if (loaded - it == STAGES - 1)
        wait_vmcnt<(STAGES - 2) * NLOADS>();
      else
        wait_vmcnt<0>();
      wait_lgkmcnt0();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      if (loaded < nk) load_next();
      __builtin_amdgcn_sched_barrier(0);
      multiply(acc, (const char*)smem + slot * SLICE_BYTES, wm, wn, lane);
      if (sum != nullptr && it % kFlush == kFlush - 1) flush(acc, sum);
      slot = slot + 1 == STAGES ? 0 : slot + 1;
    }
    wait_lgkmcnt0();
    __builtin_amdgcn_s_barrier();
  }
};

// ---------------------------------------------------------------------------
// Workgroup -> tile mapping.  Workgroups are dispatched to the 8 XCDs round
// robin (workgroup i on XCD i % 8) and each XCD has its own L2, so consecutive
// logical tile ids are handed to the workgroups of one XCD: the tiles an XCD
// runs at the same time then share operand panels in its L2.
__device__ __forceinline__ int xcd_logical(int bid, int n) {
  constexpr int X = 8;
  const int q = n / X, r = n % X;
  const int xcd = bid % X, local = bid / X;
  return xcd < r ? xcd * (q + 1) + local : r * (q + 1) + (xcd - r) * q + local;
}

// Logical id -> (mt, nt) in column-major groups of GM tile rows, so that a run
// of consecutive ids covers a GM x (run/GM) block of output tiles.
__device__ __forceinline__ void grouped_tile(int logical, int n_m, int n_n, int GM, int& mt,
                                             int& nt) {
  const int per_group = GM * n_n;
  const int group = logical / per_group;
  const int first = group * GM;
  const int gm = min(n_m - first, GM);
  const int in = logical - group * per_group;
  mt = first + in % gm;
  nt = in / gm;
}

// ---------------------------------------------------------------------------
// Online-softmax state merge in the base-2 domain (m is a running maximum of
// y*log2(e), s = sum 2^(y*log2e - m)).  An empty state is (-inf, 0); merging two of
// them stays empty.  While logits are folded an empty state is (kNoLogit, 0): logits of
// minus infinity (or whose scaled value overflows to it) then add 2^-inf = 0 to it, where
// a running maximum of -inf would make them NaN or infinite.
constexpr float kNoLogit = -3.402823466e38f;  // the lowest float32
__device__ __forceinline__ void merge_state(float& m, float& s, float mo, float so) {
  const float M = fmaxf(m, mo);
  const float ref = M == -INFINITY ? 0.f : M;
  s = s * __builtin_amdgcn_exp2f(m - ref) + so * __builtin_amdgcn_exp2f(mo - ref);
  m = M;
}

// Folds the partial states of `n` splits of token t, LPT consecutive lanes per token:
// lane l of them takes splits l, l + LPT, ... in visiting order, then the lanes merge.
// Every lane of the group ends with the whole state.
template <int LPT>
__device__ __forceinline__ void merge_splits(const float* __restrict__ mp,
                                             const float* __restrict__ sp, int64_t T, int64_t t,
                                             int n, float& m, float& s) {
  m = -INFINITY;
  s = 0.f;
#pragma unroll 4
  for (int k = threadIdx.x % LPT; k < n; k += LPT)
    merge_state(m, s, mp[(int64_t)k * T + t], sp[(int64_t)k * T + t]);
#pragma unroll
  for (int o = 1; o < LPT; o <<= 1) {
    const float mo = __shfl_xor(m, o), so = __shfl_xor(s, o);
    merge_state(m, s, mo, so);
  }
}
// Lanes per token of the merges: with many splits (few tokens) one thread per token
// would walk them serially on a nearly idle chip (32 splits at T = 256: 10.8 us).
constexpr int kManySplits = 16;

// Folds a logits tile into this lane's running states, column block by column block.
// Tiles past the end of a shard mask their padded rows; full tiles (all but the last of
// each shard) take the select-free loops.  Register r of row block i holds tile row
// wm + 32 i + acc_row(r, lane) = wm + 4 (lane / 32) + (a constant), so the mask compares
// that constant with one per-lane limit.
template <int MB, int NB>
__device__ __forceinline__ void fold_tile(const f32x16_t (&acc)[MB][NB], bool full, int lim,
                                          float (&m_run)[NB], float (&s_run)[NB]) {
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    // The maximum is taken on the raw logits and scaled once: scaling by a positive
    // constant is monotone under rounding, so this equals the maximum of the scaled
    // values.
    float tmax = -INFINITY;
    if (full) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, acc[i][j][r]);
    } else {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * i + 8 * (r >> 2) + (r & 3) < lim) tmax = fmaxf(tmax, acc[i][j][r]);
    }
    tmax *= kLog2e;
    const float scale = tmax > m_run[j] ? __builtin_amdgcn_exp2f(m_run[j] - tmax) : 1.f;
    m_run[j] = fmaxf(m_run[j], tmax);
    float sum = 0.f;
    if (full) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r], kLog2e, -m_run[j]));
    } else {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r], kLog2e, -m_run[j]));
          sum += (32 * i + 8 * (r >> 2) + (r & 3) < lim) ? e : 0.f;
        }
    }
    s_run[j] = s_run[j] * scale + sum;
  }
}

// Target gather of column block j: exactly one tile in the whole vocabulary holds a
// token's target; the lane that owns that element stores the logit.  relw: the
// target's row in this wave's WM rows (outside them: not here).
template <int MB, int NB>
__device__ __forceinline__ void gather_target(const f32x16_t (&acc)[MB][NB], int j, int64_t rel,
                                              int rows, int wm, int lane, float* y, int n) {
  if (rel >= 0 && rel < rows) {
    const int relw = (int)rel - wm;
    if (relw >= 0 && relw < 32 * MB) {
      const int rib = relw & 31;
      if (((rib >> 2) & 1) == (lane >> 5)) {
        const int want_i = relw >> 5, want_r = (rib >> 3) * 4 + (rib & 3);
        float yv = 0.f;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) yv = (i == want_i && r == want_r) ? acc[i][j][r] : yv;
        y[n] = yv;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Tile configurations.  Both element types: the direct-to-LDS ring (128-byte
// slice rows: 64 bfloat16 or 32 float32 k values, two slots) with 256 x 256
// tiles; LogitsTail is the same tile for a d that is not a multiple of the slice
// depth (a kernel of its own, so that the per-lane addresses of the last slice cost
// the usual widths no registers).
template <class E> struct Cfg;
template <> struct Cfg<Bf16> {
  // 512-thread workgroups (two wavefronts per SIMD), 256 x 256 tiles, 128 x 64 per
  // wave, for every contraction (measured faster inside the backward stage launch
  // than 256 x 192 tiles with 64 x 96 per wave, whose fragment reads per MFMA are
  // higher).  One wavefront per SIMD with 128 x 128 per wave reads a third less LDS
  // per MFMA and runs at a higher clock, but measured 5-17% slower: a lone wave's
  // load waits and barrier waits idle the MFMA pipe.
  using Logits = GemmDma<256, 256, 2, 4>;
  using Mm = Logits;  // the dH / dW contractions
  // the last dH / dW column block when d leaves 1..64 columns past a multiple of
  // 256 (160 x 64 per wave, 0.7 fragment reads per MFMA)
  using MmWide = GemmDma<320, 256, 2, 4>;
  using LogitsTail = GemmDma<256, 256, 2, 4, Bf16, true>;
  using Stream128 = Ring<256, 128, 4, 2, 3, Bf16>;  // forward on few tokens, see fwd_tile
  using Stream64 = Ring<128, 64, 4, 2, 6, Bf16>;
  // The backward's tile classes (StageArgs): 0: Logits, Tr256, Tr320; 1: Res128x64,
  // Tr128x64; 2: Res128, Tr128; 3: Logits, Mm, MmWide.  Measured, backward alone (us,
  // classes 0 / 1 / 2): bf16 T = 2048, d = 2880, V = 201088 6661 / 9770 / 8406 and T = 40,
  // d = 1000, V = 32003 98 / 74 / 76; float32 T = 256, d = 256, V = 2048 153 / 47 / 62 and
  // T = 2048, d = 2880, V = 50000 13961 / 13173 / 13273; class 3 against 0: bf16 T = 32768,
  // d = 2880, V = 201088 96.3 against 97.1 ms, T = 4096 12.60 against 12.38 ms.
  using Tr256 = GemmDma<256, 256, 2, 4, Bf16, false, true>;
  using Tr320 = GemmDma<320, 256, 2, 4, Bf16, false, true>;
  using Res128 = GemmDma<128, 128, 2, 2, Bf16, true>;
  using Tr128 = GemmDma<128, 128, 2, 2, Bf16, false, true>;
  using Res128x64 = Ring<128, 64, 4, 2, 3, Bf16>;
  using Tr128x64 = Ring<128, 64, 4, 2, 3, Bf16, true>;
};
template <> struct Cfg<F32> {
  // The same direct-to-LDS ring and 256 x 256 tiles: 32 float32 k values per slice,
  // four 32x32x2 f32 MFMAs per fragment pair.
  using Logits = GemmDma<256, 256, 2, 4, F32>;
  using LogitsTail = GemmDma<256, 256, 2, 4, F32, true>;
  using Stream128 = Ring<256, 128, 4, 2, 3, F32>;
  using Stream64 = Ring<128, 64, 4, 2, 6, F32>;
  using Mm = Logits;
  using MmWide = GemmDma<320, 256, 2, 4, F32>;
  using Res128 = GemmDma<128, 128, 2, 2, F32, true>;
  using Tr128 = GemmDma<128, 128, 2, 2, F32, false, true>;
  using Res128x64 = Ring<128, 64, 4, 2, 3, F32>;
  using Tr128x64 = Ring<128, 64, 4, 2, 3, F32, true>;
};

static inline bool launched_ok() { return hipGetLastError() == hipSuccess; }

}  // namespace vpce
