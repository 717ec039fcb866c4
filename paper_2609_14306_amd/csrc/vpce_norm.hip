// Layer norm of the hidden states and its gradients, for gfx950 (MI355X).
//
// Both directions are bound by memory: the forward reads X and writes Y once (2 e T d
// bytes for elements of e bytes), the backward reads X and dY and writes dX once
// ((e + 8) T d bytes).  So a row is loaded once and stays in registers, spread over W
// wavefronts with a few 16-byte vectors of X in each lane; its sums are taken from there.
// The variance is a second sum over the registers, around the mean, not a difference of
// squares.  A float32 mean far above the spread is itself some roundings off, which the
// spread would see: in a row whose mean is more than 4 spreads away the distances' own mean
// (`left`, a third sum: 1% of the time, T = 32768, d = 2880) takes what is left of it out of
// Y, rstd and the stored mean; nearer ones have roundings of the mean no larger than those of
// the distances.  The backward has the mean in float32 alone: one rounding of it is what xh of
// such a row is off by there.
//
// MI355X, kernels alone, averages: T = 32768, d = 2880, bfloat16 forward 74 us (5.1 TB/s; 69.2
// among others of its kind), backward 172 + 4.8 us (5.5 TB/s); T = 16384, d = 7168, float32
// without a mean 165 us (5.7 TB/s) and 263 + 4.8 us (5.4 TB/s); a 1 GiB copy runs at 5.1 TB/s.
// With a residual (X + R stored and normalised; dS added in the backward), bfloat16 without a mean:
// T = 32768, d = 2880 with the result in 8 bits 120 us (7 bytes an element, 5.5 TB/s), backward T = 16384,
// d = 7168 301 + 5 us (14 bytes, 5.5 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "vpce_f8.h"
#include "vpce_head.h"
#include "vpce_lanes.h"

namespace vpce {

namespace {

// Element types: VEC elements per 16 bytes, as float32 and back.
struct Half {  // bfloat16
  using storage = uint16_t;
  static constexpr int VEC = 8;
  __device__ static void unpack(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[2 * k] = __uint_as_float(w[k] << 16);
      f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
  // round to nearest even; a NaN stays a NaN
  __device__ static uint32_t pack2(float lo, float hi) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
  }
  __device__ static uint4 pack(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
  }
};
struct Single {
  using storage = float;
  static constexpr int VEC = 4;
  __device__ static void unpack(const uint4& u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
  }
  __device__ static uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

// A row spread over LANES lanes, EL elements each: a lane's share is the vectors i,
// i + LANES, ... (NV of them) of the row's nvec.  Rows of up to 64 lanes lie side by side
// in the wavefronts of a workgroup of 256.
template <class E, int LANES_, int EL>
struct Row {
  static constexpr int LANES = LANES_, VEC = E::VEC, NV = EL / VEC;
  static constexpr int W = LANES > 64 ? LANES / 64 : 1;
  static constexpr int ROWS = LANES <= 64 ? 256 / LANES : 1;  // rows of a workgroup at a time
  static constexpr int NT = LANES * ROWS;
};

// Sums N values over the LANES lanes of a row, the same bits in each.  red holds two
// sets, taken in turn (`turn`), so that one barrier a sum is enough: a set is written
// again only behind the next sum's barrier.
template <int LANES, int N, int W>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*red)[N][W], int& turn) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] += lane_move<kSwap1>(v[k]);
    v[k] += lane_move<kSwap2>(v[k]);
    v[k] += lane_move<kHalfMirror>(v[k]);
    if constexpr (LANES >= 16) v[k] += lane_move<kMirror>(v[k]);
    if constexpr (LANES == 32) v[k] += __shfl_xor(v[k], 16);
    if constexpr (LANES >= 64)
      v[k] = (lane_read(v[k], 0) + lane_read(v[k], 16)) + (lane_read(v[k], 32) + lane_read(v[k], 48));
  }
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) red[turn][k][threadIdx.x >> 6] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = red[turn][k][0];
#pragma unroll
      for (int w = 1; w < W; ++w) v[k] += red[turn][k][w];
    }
    turn ^= 1;
  }
}

// The row y in 8 bits: the lanes that share 128 columns find their largest magnitude, and with it
// the scale.  A block is 128 / VEC consecutive vectors, i.e. as many lanes, or the LANES of a narrow
// row with all their vectors.
template <class E, int LANES, int EL>
__device__ __forceinline__ void store_f8(const NormArgs& a, int64_t t, int lane, const float (&y)[EL / E::VEC][E::VEC]) {
  constexpr int VEC = E::VEC, NV = EL / VEC;
  constexpr int GRP = LANES < 128 / VEC ? LANES : 128 / VEC;
  constexpr int KS = GRP < 128 / VEC ? NV : 1;  // vectors of a lane in a block
  static_assert(GRP == 128 / VEC || LANES * EL <= 128, "a block is whole in its lanes");
  const int nvec = a.d / VEC, nb = (a.d + 127) / 128;
#pragma unroll
  for (int k0 = 0; k0 < NV; k0 += KS) {
    float m = 0.f;
#pragma unroll
    for (int k = k0; k < k0 + KS; ++k)
      if (lane + k * LANES < nvec)
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = fmaxf(m, finite_magnitude(y[k][j]));
    const int b = f8_scale(lanes_max<GRP>(m));
    const float inverse = f8_inverse(b);
#pragma unroll
    for (int k = k0; k < k0 + KS; ++k) {
      const int i = lane + k * LANES;
      if (i >= nvec) continue;
      uint32_t* out = (uint32_t*)(a.Y8 + t * a.d) + i * (VEC / 4);
      uint32_t w[VEC / 4];
#pragma unroll
      for (int q = 0; q < VEC / 4; ++q)
        w[q] = f8_pack4(y[k][4 * q] * inverse, y[k][4 * q + 1] * inverse, y[k][4 * q + 2] * inverse,
                        y[k][4 * q + 3] * inverse);
      if constexpr (VEC == 8)
        *(uint2*)out = make_uint2(w[0], w[1]);
      else
        *out = w[0];
    }
    const int i = lane + k0 * LANES;
    if (lane % GRP == 0 && i < nvec) a.scale[t * nb + i / (128 / VEC)] = (uint8_t)b;
  }
}

// ADD: X + R, rounded, is stored and normalised, and y may leave in 8 bits.
template <class E, bool RMS, int LANES, int EL, bool ADD>
__global__ void __launch_bounds__((Row<E, LANES, EL>::NT)) norm_forward_kernel(NormArgs a) {
  using R = Row<E, LANES, EL>;
  constexpr int VEC = R::VEC, NV = R::NV;
  __shared__ float red[2][1][R::W];
  const int lane = threadIdx.x % R::LANES, nvec = a.d / VEC;
  const int64_t t = (int64_t)blockIdx.x * R::ROWS + threadIdx.x / R::LANES;
  if (R::ROWS > 1 && t >= a.T) return;  // (such rows have no barriers)
  const uint4* x = (const uint4*)a.X + t * nvec;
  uint4* y = (uint4*)a.Y + t * nvec;
  int turn = 0;

  float f[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = lane + k * R::LANES;
    E::unpack(i < nvec ? x[i] : make_uint4(0, 0, 0, 0), f[k]);
    if constexpr (ADD) {
      float r[VEC];
      E::unpack(i < nvec ? ((const uint4*)a.R + t * nvec)[i] : make_uint4(0, 0, 0, 0), r);
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[k][j] += r[j];
      const uint4 sum = E::pack(f[k]);
      if (i < nvec) ((uint4*)a.S + t * nvec)[i] = sum;
      E::unpack(sum, f[k]);
    }
  }
  const float inv_d = 1.f / (float)a.d;
  float mean = 0.f, left = 0.f;
  if (!RMS) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[0] += f[k][j];
    row_sum<LANES>(s, red, turn);
    mean = s[0] * inv_d;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const bool in = lane + k * R::LANES < nvec;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      if (!RMS) f[k][j] = in ? f[k][j] - mean : 0.f;
      s[0] = __builtin_fmaf(f[k][j], f[k][j], s[0]);
    }
  }
  row_sum<LANES>(s, red, turn);
  float var = s[0] * inv_d;
  if (!RMS && mean * mean > 16.f * var) {  // (the same for every lane of the row)
    float c[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < VEC; ++j) c[0] += f[k][j];
    row_sum<LANES>(c, red, turn);
    left = c[0] * inv_d;
    var = __builtin_fmaf(-left, left, var);
    var = var < 0.f ? 0.f : var;
  }
  const float rstd = 1.f / sqrtf(var + a.eps), shift = -left * rstd;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = lane + k * R::LANES;
    if (i < nvec) {
      float ga[VEC], be[VEC];
      E::unpack(((const uint4*)a.gamma)[i], ga);
      if (a.beta) E::unpack(((const uint4*)a.beta)[i], be);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float xh = RMS ? f[k][j] * rstd : __builtin_fmaf(f[k][j], rstd, shift);
        ga[j] = a.beta ? __builtin_fmaf(xh, ga[j], be[j]) : xh * ga[j];
        if constexpr (ADD) f[k][j] = ga[j];
      }
      if (!ADD || a.Y) y[i] = E::pack(ga);
    }
  }
  if constexpr (ADD)
    if (a.Y8) store_f8<E, LANES, EL>(a, t, lane, f);
  if (lane == 0) {
    a.rstd[t] = rstd;
    if (!RMS) a.mean[t] = mean + left;
  }
}

// One workgroup walks rows blockIdx.x, + gridDim.x, ... (ROWS side by side where a row
// is a single wavefront) with the sums of dgamma and dbeta over them in registers, and
// leaves these as one row of partial sums each (or the result, where it is alone).  The
// order of every sum depends on the sizes alone: the same call gives the same bits.
template <class E, bool RMS, int LANES, int EL, bool ADD>
__global__ void __launch_bounds__((Row<E, LANES, EL>::NT)) norm_backward_kernel(NormGradArgs a) {
  using R = Row<E, LANES, EL>;
  constexpr int VEC = R::VEC, NV = R::NV;
  // the next row is loaded while this one is reduced, where there are registers for it
  constexpr bool AHEAD = EL * LANES <= 8192;
  __shared__ float red[2][2][R::W];
  const int lane = threadIdx.x % R::LANES, group = threadIdx.x / R::LANES, nvec = a.d / VEC;
  const int64_t step = (int64_t)gridDim.x * R::ROWS;
  const float inv_d = 1.f / (float)a.d;
  int turn = 0;

  uint4 ga[NV];
  float dg[NV][VEC], db[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int i = lane + k * R::LANES;
    ga[k] = i < nvec ? ((const uint4*)a.gamma)[i] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dg[k][j] = db[k][j] = 0.f;
  }
  uint4 xn[NV];
  // (dS of the next row, too; without AHEAD it is read where it is added)
  float4 dyn[NV][VEC / 4], dsn[ADD && AHEAD ? NV : 1][VEC / 4];
  float mean_n = 0.f, rstd_n = 0.f;
  auto load = [&](int64_t t) {
    if (t >= a.T) return;
    const uint4* x = (const uint4*)a.X + t * nvec;
    const float4* dy = (const float4*)a.dY + t * (a.d / 4);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = lane + k * R::LANES;
      if (i < nvec) {
        xn[k] = x[i];
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
          dyn[k][q] = dy[i * (VEC / 4) + q];
          if constexpr (ADD && AHEAD) dsn[k][q] = ((const float4*)a.dS + t * (a.d / 4))[i * (VEC / 4) + q];
        }
      }
    }
    if (!RMS) mean_n = a.mean[t];
    rstd_n = a.rstd[t];
  };
  int64_t t = (int64_t)blockIdx.x * R::ROWS + group;
  if (AHEAD) load(t);
  for (; t < a.T; t += step) {
    if (!AHEAD) load(t);
    uint4 xr[NV];
    float dy[NV][VEC];
    float4 ds[ADD && AHEAD ? NV : 1][VEC / 4];
    const float mean = mean_n, rstd = rstd_n;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      xr[k] = xn[k];
#pragma unroll
      for (int q = 0; q < VEC / 4; ++q) {
        if constexpr (ADD && AHEAD) ds[k][q] = dsn[k][q];
        dy[k][4 * q] = dyn[k][q].x;
        dy[k][4 * q + 1] = dyn[k][q].y;
        dy[k][4 * q + 2] = dyn[k][q].z;
        dy[k][4 * q + 3] = dyn[k][q].w;
      }
    }
    if (AHEAD) load(t + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (lane + k * R::LANES < nvec) {
        float x[VEC], g[VEC];
        E::unpack(xr[k], x);
        E::unpack(ga[k], g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float xh = (x[j] - mean) * rstd, gy = g[j] * dy[k][j];
          s[0] += gy;
          s[1] = __builtin_fmaf(gy, xh, s[1]);
          dg[k][j] = __builtin_fmaf(dy[k][j], xh, dg[k][j]);
          db[k][j] += dy[k][j];
        }
      }
    row_sum<LANES>(s, red, turn);
    const float c1 = RMS ? 0.f : s[0] * inv_d, c2 = s[1] * inv_d;
    float4* dx = (float4*)a.dX + t * (a.d / 4);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = lane + k * R::LANES;
      if (i < nvec) {
        float x[VEC], g[VEC];
        E::unpack(xr[k], x);
        E::unpack(ga[k], g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float xh = (x[j] - mean) * rstd;
          g[j] = rstd * (g[j] * dy[k][j] - c1 - xh * c2);
          if constexpr (ADD && AHEAD) g[j] += ((const float*)&ds[k][j / 4])[j % 4];
        }
        if constexpr (ADD && !AHEAD)
#pragma unroll
          for (int q = 0; q < VEC / 4; ++q) {
            const float4 s4 = ((const float4*)a.dS + t * (a.d / 4))[i * (VEC / 4) + q];
            g[4 * q] += s4.x;
            g[4 * q + 1] += s4.y;
            g[4 * q + 2] += s4.z;
            g[4 * q + 3] += s4.w;
          }
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q)
          dx[i * (VEC / 4) + q] = make_float4(g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]);
      }
    }
  }

  // the rows side by side first
  if constexpr (R::ROWS > 1) {
    __shared__ float side[R::ROWS][R::LANES][2 * VEC + 1];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        side[group][lane][j] = dg[k][j];
        side[group][lane][VEC + j] = db[k][j];
      }
      __syncthreads();
      if (group == 0)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
#pragma unroll
          for (int r = 1; r < R::ROWS; ++r) {
            dg[k][j] += side[r][lane][j];
            db[k][j] += side[r][lane][VEC + j];
          }
      __syncthreads();
    }
    if (group > 0) return;
  }
  const bool alone = gridDim.x == 1;
  float* out[2] = {alone ? a.dgamma : a.part + (int64_t)blockIdx.x * a.d,
                   alone ? a.dbeta : a.part + ((int64_t)gridDim.x + blockIdx.x) * a.d};
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    if (p == 1 && !a.dbeta) break;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int i = lane + k * R::LANES;
      if (i < nvec)
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
          const float(&v)[VEC] = p ? db[k] : dg[k];
          float4* o = (float4*)out[p] + i * (VEC / 4) + q;
          float4 w = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          if (alone && a.accumulate) {
            const float4 old = *o;
            w = make_float4(old.x + w.x, old.y + w.y, old.z + w.z, old.w + w.w);
          }
          *o = w;
        }
    }
  }
}

// dgamma (blockIdx.y 0) and dbeta (1) from n rows of partial sums: 64 columns a
// workgroup, sixteen wavefronts side by side down the rows.
__global__ void __launch_bounds__(1024) norm_weight_grad_kernel(NormGradArgs a, int n) {
  __shared__ float side[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = blockIdx.x * 64 + lane;
  const float* part = a.part + (int64_t)blockIdx.y * n * a.d;
  float v = 0.f;
  if (j < a.d)
#pragma unroll 8
    for (int r = wave; r < n; r += 16) v += part[(int64_t)r * a.d + j];
  side[wave][lane] = v;
  __syncthreads();
  if (wave > 0 || j >= a.d) return;
  for (int w = 1; w < 16; ++w) v += side[w][lane];
  float* out = blockIdx.y ? a.dbeta : a.dgamma;
  out[j] = a.accumulate ? out[j] + v : v;
}

bool launched_ok() { return hipGetLastError() == hipSuccess; }

// Run f.run<LANES, EL>() for the layout of a row of d elements.
//
// Forward: 32 bytes of X a lane (64 for bfloat16 rows of 2049 to 3456 elements).  Fewer
// bytes a lane leave more of a workgroup to its two sums, more leave fewer loads in
// flight, and what counts as few differs by type.  GB/s, bfloat16 / float32:
//   T = 65536, d = 1000: 64 x 16 5520 / 5020, 128 x 8 4720 / 5630
//   T = 30000, d = 2048: 128 x 16 5430 / 5610, 256 x 8 4710 / 5860
//   T = 32768, d = 2880: 128 x 32 5480 / 5480, 256 x 16 5270 / 5870, 512 x 8 4050 / 6010
//   T = 32768, d = 3456: 128 x 32 5380, 256 x 16 5340 (bfloat16; without a mean 5720, 5830)
//   T = 16384, d = 3584: 128 x 32 4990, 256 x 16 5220 (bfloat16)
//   T = 16384, d = 4096: 128 x 32 5320 / 5370, 256 x 16 5530 / 5730, 512 x 8 4860 / 5950
//   T = 16384, d = 7168: 256 x 32 5240 / 5480, 512 x 16 5330 / 5790, 1024 x 8 4440 / 5880
// With few rows fewer bytes a lane win (bfloat16, d = 4096, 128 x 32 and 256 x 16: T = 1 3.2 and
// 2.7 us, T = 512 4.3 and 3.8; T = 4096, which the cache holds, 12.6 and 13.5).
// With a residual there are four streams instead of two, and 256 x 16 takes the widths of 128 x 32
// (T = 32768, d = 2880, bfloat16: 116 us instead of 126 with the result in 8 bits, 128 instead of 135
// without; the other layouts stay the fastest ones or within 2%).
template <class E, bool ADD, class F>
bool forward_layout(int d, F&& f) {
  if (d <= 64) return f.template run<8, 8>();
  if (d <= 128) return f.template run<16, 8>();
  if (d <= 256) return f.template run<32, 8>();
  if (d <= 512) return f.template run<64, 8>();
  if constexpr (E::VEC == 8) {
    if (d <= 1024) return f.template run<64, 16>();
    if (d <= 2048) return f.template run<128, 16>();
    if (!ADD && d <= 3456) return f.template run<128, 32>();
    if (d <= 4096) return f.template run<256, 16>();
    if (d <= 8192) return f.template run<512, 16>();
  } else {
    if (d <= 1024) return f.template run<128, 8>();
    if (d <= 2048) return f.template run<256, 8>();
    if (d <= 4096) return f.template run<512, 8>();
    if (d <= 8192) return f.template run<1024, 8>();
  }
  return f.template run<1024, 16>();
}

// Backward: as few wavefronts as hold the row with its sums and the next row in registers.
template <class F>
bool backward_layout(int d, F&& f) {
  if (d <= 64) return f.template run<8, 8>();
  if (d <= 128) return f.template run<16, 8>();
  if (d <= 256) return f.template run<32, 8>();
  if (d <= 512) return f.template run<64, 8>();
  if (d <= 1024) return f.template run<64, 16>();
  if (d <= 2048) return f.template run<256, 8>();
  if (d <= 4096) return f.template run<256, 16>();
  if (d <= 8192) return f.template run<512, 16>();
  return f.template run<1024, 16>();
}

template <class E, bool RMS, bool ADD>
struct Forward {
  const NormArgs& a;
  hipStream_t s;
  // A launch takes at most 2^30 threads (its size is a 32-bit number of threads: 2^23 rows
  // of 1024 would not fit), and further rows further launches.
  template <int LANES, int EL>
  bool run() {
    using R = Row<E, LANES, EL>;
    constexpr int64_t kRows = (int64_t)R::ROWS * ((1 << 30) / R::NT);
    for (int64_t t = 0; t < a.T; t += kRows) {
      NormArgs b = a;
      b.T = std::min(kRows, a.T - t);
      using S = typename E::storage;
      b.X = (const S*)a.X + t * a.d;
      b.Y = a.Y ? (S*)a.Y + t * a.d : nullptr;
      b.mean = RMS ? nullptr : a.mean + t;
      b.rstd = a.rstd + t;
      if constexpr (ADD) {
        b.R = (const S*)a.R + t * a.d;
        b.S = (S*)a.S + t * a.d;
        b.Y8 = a.Y8 ? a.Y8 + t * a.d : nullptr;
        b.scale = a.Y8 ? a.scale + t * ((a.d + 127) / 128) : nullptr;
      }
      hipLaunchKernelGGL((norm_forward_kernel<E, RMS, LANES, EL, ADD>),
                         dim3((unsigned)((b.T + R::ROWS - 1) / R::ROWS)), dim3(R::NT), 0, s, b);
      if (!launched_ok()) return false;
    }
    return true;
  }
};

template <class E, bool RMS, bool ADD>
struct Backward {
  const NormGradArgs& a;
  hipStream_t s;
  template <int LANES, int EL>
  bool run() {
    using R = Row<E, LANES, EL>;
    const int n = norm_parts(a.T, a.d);
    hipLaunchKernelGGL((norm_backward_kernel<E, RMS, LANES, EL, ADD>), dim3((unsigned)n), dim3(R::NT), 0, s, a);
    if (!launched_ok()) return false;
    if (n == 1) return true;
    hipLaunchKernelGGL(norm_weight_grad_kernel, dim3((unsigned)((a.d + 63) / 64), a.dbeta ? 2u : 1u), dim3(1024), 0, s,
                       a, n);
    return launched_ok();
  }
};

// Workgroups of a backward, each with one row of partial sums.  Rows are walked by one
// workgroup a CU, or two where a workgroup's rows hold 2048 elements: with the next row on
// its way that keeps the memory busy, and more of them only add partial sums to write and
// read (T = 32768, d = 2880, bfloat16: 256 workgroups 171 us, 512 173, 1024 196; float32
// 195, 212, 231; T = 30000, d = 1200: 113, 75, 72 and 110, 80, 84).  No workgroup sums more
// than 1024 rows in one chain.  Up to four rounds of rows one workgroup does it all and
// the second launch is saved (d = 4096, us a call: T = 4 so 7.7, T = 5 in two launches 11.0;
// T = 16 in one workgroup took 20.4, 8 as long as in two).
struct Parts {
  int rows, n;
  template <int LANES, int EL>
  bool run() {
    rows = Row<Half, LANES, EL>::ROWS;
    n = LANES * EL * rows == 2048 ? 512 : 256;
    return true;
  }
};

}  // namespace

int norm_parts(int64_t T, int d) {
  Parts p{};
  backward_layout(d, p);
  const int64_t rounds = (T + p.rows - 1) / p.rows;
  if (rounds <= 4) return 1;
  return (int)std::max<int64_t>(std::min<int64_t>(rounds, p.n), (rounds + 1023) / 1024);
}

template <bool RMS, bool ADD>
static bool forward_of(int dtype, const NormArgs& a, hipStream_t s) {
  return dtype == VP_BF16 ? forward_layout<Half, ADD>(a.d, Forward<Half, RMS, ADD>{a, s})
                          : forward_layout<Single, ADD>(a.d, Forward<Single, RMS, ADD>{a, s});
}
bool run_norm_forward(int dtype, bool rms, const NormArgs& a, hipStream_t s) {
  if (a.R) return rms ? forward_of<true, true>(dtype, a, s) : forward_of<false, true>(dtype, a, s);
  return rms ? forward_of<true, false>(dtype, a, s) : forward_of<false, false>(dtype, a, s);
}
template <bool RMS, bool ADD>
static bool backward_of(int dtype, const NormGradArgs& a, hipStream_t s) {
  return dtype == VP_BF16 ? backward_layout(a.d, Backward<Half, RMS, ADD>{a, s})
                          : backward_layout(a.d, Backward<Single, RMS, ADD>{a, s});
}
bool run_norm_backward(int dtype, bool rms, const NormGradArgs& a, hipStream_t s) {
  if (a.dS) return rms ? backward_of<true, true>(dtype, a, s) : backward_of<false, true>(dtype, a, s);
  return rms ? backward_of<true, false>(dtype, a, s) : backward_of<false, false>(dtype, a, s);
}

}  // namespace vpce
