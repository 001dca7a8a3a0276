// The gated feed-forward projections and their gradients.
//
//   g_t = Wg x_t,  u_t = Wu x_t,  h_t = act(g_t) u_t
// and for a gradient dh
//   dg = dh u act'(g),  du = dh act(g),
//   dx = Wg^T dg + Wu^T du,  dWg = sum_t dg_t x_t^T,  dWu = sum_t du_t x_t^T.
//
// Forward: one product whose tiles hold the same columns of Wg and of Wu (PAIR in product.h), so that g and u
// of a value of h meet in one lane's registers, and the activation and the product are its epilogue: g and u
// never reach memory.  Backward: the same product again, whose epilogue reads dh and writes d = (dg | du); x is
// all that it needs of the forward, and g and u are those of 32 bits, not a rounding of them kept from one pass to
// the other (which would take 4 f bytes a row over that time, and exactness from d).  dx is one product of d's rows
// with the weights' columns, and dW one of d's columns with x's: x, and past 192 rows the weights, are transposed
// first (prepare_kernel), d is written both ways round by the epilogue.
#include "checkpoint.h"
#include "common.h"
#include "half.h"
#include "kernels.h"
#include "product.h"
#include "tiles.h"

namespace hpr {

namespace {

// ---- activations ------------------------------------------------------------------------------

// exp of a 32-bit number, relative error (|x| + 2) 2^-24: far below the rounding of what it goes into.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

struct Silu {
  // (exp overflows to infinity below -88, where the value is 0 to within 1e-36)
  static __device__ __forceinline__ float sigmoid(float g) {
    return __builtin_amdgcn_rcpf(1.f + exp_of(-g));
  }
  static __device__ __forceinline__ float value(float g) { return g * sigmoid(g); }
  static __device__ __forceinline__ void both(float g, float& v, float& slope) {
    const float s = sigmoid(g);
    v = g * s;
    slope = s * (1.f + g * (1.f - s));
  }
};

// g Phi(g), Phi(-x sqrt 2) = erfc(x) / 2 = exp(-x^2) t P(t) with t = 1 / (1 + 0.4 x), x >= 0: erfc(x) exp(x^2) / t
// is smooth on (0, 1], and P, of degree 8, is a least-squares fit to it with the weights moved towards the largest
// relative error; in 32 bits within 2.7e-7 of it, in the tail too (h of 13,057 rows, 768 -> 2304 in fp16: 108 us
// with it, 130 with the library's erfc).
struct Gelu {
  static __device__ __forceinline__ float cdf(float g, float& e) {
    const float t = __builtin_amdgcn_rcpf(1.f + __builtin_fabsf(g) * (0.4f * 0.70710678f));
    e = exp_of(-0.5f * g * g);
    constexpr float c[9] = {0.22567586600780487f,  0.22566956281661987f, 0.20784330368041992f,
                            0.16853772103786469f,  0.14144709706306458f, -0.005639823153614998f,
                            0.16912293434143066f,  -0.18292437493801117f, 0.05026784539222717f};
    float p = c[8];
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __builtin_fmaf(p, t, c[i]);
    const float q = 0.5f * t * p * e;
    return g < 0.f ? q : 1.f - q;
  }
  static __device__ __forceinline__ float value(float g) {
    float e;
    return g * cdf(g, e);
  }
  static __device__ __forceinline__ void both(float g, float& v, float& slope) {
    float e;
    const float p = cdf(g, e);
    v = g * p;
    slope = p + g * 0.39894228f * e;
  }
};

// g (1 + tanh z) / 2 = g / (1 + exp(-2 z)), z = sqrt(2 / pi) (g + 0.044715 g^3)
struct GeluTanh {
  static __device__ __forceinline__ float part(float g) {
    return __builtin_amdgcn_rcpf(1.f + exp_of(-1.59576912f * g * (1.f + 0.044715f * g * g)));
  }
  static __device__ __forceinline__ float value(float g) { return g * part(g); }
  static __device__ __forceinline__ void both(float g, float& v, float& slope) {
    const float s = part(g);
    v = g * s;
    // (s (1 - s) is 0 in 32 bits long before g^2 passes them)
    const float q = s * (1.f - s);
    slope = s + (q > 0.f ? g * q * 1.59576912f * (1.f + 0.134145f * g * g) : 0.f);
  }
};

// ---- powers of two of fp16 --------------------------------------------------------------------

// dg and du are products' operands in 16 bits.  fp16 has few exponents: where dh is small (a loss that is
// not scaled), they would lose bits below 2^-14.  So a row of d is written for dx times the power of two that
// brings the row's largest |dh| into [1, 2), a column for dW times that of its column, and the products'
// results are multiplied back in 32 bits: exactly undone, whatever the size of dh.  What is left are factors
// act(g) and u act'(g) as small as the forward's own h, which fp16 rounds as coarsely; and they overflow where
// they pass 2^15, as a finite h all but excludes.
// bits: the largest |value| of fp16 as a whole number (max_kernel); 0 and infinities stay as they are.
__device__ __forceinline__ int up_of(uint32_t bits) {
  if (bits == 0 || bits >= 0x7c00) return 0;
  const float v = (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  return 127 - (int)(__float_as_uint(v) >> 23);
}
__device__ __forceinline__ float power_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Largest |dh| of every row and column: 4 ROWS rows of 512 columns per workgroup, a row per wave at a time, four on
// their way.  The maxima of workgroups meet in atomic maxima of whole numbers, which have no order.
template <int ROWS>
__global__ __launch_bounds__(256) void max_kernel(const uint16_t* dh, int64_t n, int f, uint32_t* rows,
                                                  uint32_t* cols) {
  __shared__ uint32_t part[4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t n_c = (uint32_t)(f + 511) / 512u;
  const int c = (int)(blockIdx.x % n_c) * 512 + 8 * lane;
  const int64_t t0 = (int64_t)(blockIdx.x / n_c) * (4 * ROWS) + wave * ROWS;
  uint32_t most[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 1
  for (int i = 0; i < ROWS; i += 4) {
    u32x4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = u32x4{0u, 0u, 0u, 0u};
      if (c < f && t0 + i + q < n) v[q] = load16(dh + (t0 + i + q) * f + c);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t row = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t b = (v[q][e >> 1] >> (16 * (e & 1))) & 0x7fffu;
        most[e] = most[e] > b ? most[e] : b;
        row = row > b ? row : b;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)row, d);
        row = row > o ? row : o;
      }
      if (lane == 0 && t0 + i + q < n) atomicMax(rows + t0 + i + q, row);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[wave][8 * lane + e] = most[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += 256) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = m > part[w][i] ? m : part[w][i];
    const int col = (int)(blockIdx.x % n_c) * 512 + i;
    if (col < f) atomicMax(cols + col, m);
  }
}

// ---- h, and d -----------------------------------------------------------------------------------

// dg and du of one value.
template <class A>
__device__ __forceinline__ void gradients(float g, float u, float dh, float& dg, float& du) {
  float v, slope;
  A::both(g, v, slope);
  dg = dh * u * slope;
  du = dh * v;
}

template <class T, class A, class P, int G, bool GRAD>
__device__ __forceinline__ void gated_tile(const GatedArgs& a) {
  constexpr int kT = P::kT, kM = P::kM, kH = kM / 2;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // P::kLds
  const int lane = threadIdx.x & 63, row = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wave % P::kWt, wm = wave % P::kW / P::kWt;  // (of group 0, which stores)
  const int n_m = (a.f + P::kCols - 1) / P::kCols;
  const TileAt at = tile_at(blockIdx.x, gridDim.x, (uint32_t)((a.n + P::kRows - 1) / P::kRows), n_m);
  const int64_t t0 = (int64_t)at.t * P::kRows;
  const int m0 = at.m * P::kCols;
  const int64_t left_t = a.n - t0;
  const int last_t = left_t < P::kRows ? (int)left_t - 1 : P::kRows - 1;
  const int last_m = a.f - m0 < P::kCols ? a.f - m0 - 1 : P::kCols - 1;
  typename P::Acc acc;
  const int64_t w0 = (int64_t)m0 * a.k;
  if (!grouped<P, G>(a.x + t0 * a.x_ld, (int)a.x_ld, last_t, {{a.wg + w0, a.wu + w0}, a.k, last_m}, a.k, at, smem,
                     wave, lane, acc))
    return;

  const int mw = m0 + wm * P::kWaveCols;  // the wave's first column
  const int64_t tw = t0 + wt * kT * 16;   // and row
  constexpr int kOwn = 16 * 32 * (kH > kT ? kH : kT);
  constexpr int kSums = (G - 1) * P::kW * kM * kT * 1024;
  static_assert(kSums + P::kW * kOwn <= G * P::kLds, "the waves' blocks fit beside the sums");
  unsigned char* own = smem + kSums + wave * kOwn;
  if constexpr (!GRAD) {
#pragma unroll
    for (int j = 0; j < kT; ++j)
      store_rows16<T, kH>(a.h + (tw + 16 * j) * a.f + mw, a.f, a.n - tw - 16 * j, a.f - mw, own, lane,
                          [&](int i, int e) { return A::value(acc[i][j][e]) * acc[i + kH][j][e]; });
  } else {
    // d in the place of g and u; 0 past the last row
#pragma unroll
    for (int j = 0; j < kT; ++j) {
      const int64_t t = tw + 16 * j + row;
      uint2 w[kH];
#pragma unroll
      for (int i = 0; i < kH; ++i) {
        const int m = mw + 16 * i + 4 * q;
        w[i] = uint2{0u, 0u};
        if (t < a.n && m < a.f) w[i] = *reinterpret_cast<const uint2*>(a.dh + t * a.f + m);
      }
#pragma unroll
      for (int i = 0; i < kH; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t b = e < 2 ? w[i].x : w[i].y;
          float dg, du;
          gradients<A>(acc[i][j][e], acc[i + kH][j][e], e & 1 ? T::hi(b) : T::lo(b), dg, du);
          acc[i][j][e] = t < a.n ? dg : 0.f;
          acc[i + kH][j][e] = t < a.n ? du : 0.f;
        }
    }
    if (a.d) {
#pragma unroll
      for (int j = 0; j < kT; ++j) {
        const int64_t t = tw + 16 * j + row;
        float up = 1.f;
        if constexpr (T::kNarrow) up = power_of(up_of(a.row_max[t < a.n ? t : a.n - 1]));
#pragma unroll
        for (int s = 0; s < 2; ++s)
          store_rows16<T, kH>(a.d + (tw + 16 * j) * 2 * a.f + (int64_t)s * a.f + mw, 2 * (int64_t)a.f,
                              a.n - tw - 16 * j, a.f - mw, own, lane,
                              [&](int i, int e) { return acc[s * kH + i][j][e] * up; });
      }
    }
    if (a.dt) {  // 16 columns of d at a time, 16 kT values of each
      constexpr int kRow = 32 * kT, kCh = kRow / 16, kPer = 64 / kCh;
#pragma unroll
      for (int i = 0; i < kM; ++i) {
        const int m_first = mw + 16 * (i % kH);
        float up[4] = {1.f, 1.f, 1.f, 1.f};
        if constexpr (T::kNarrow) {
          if (m_first + 4 * q < a.f) {
            const u32x4 bits = *reinterpret_cast<const u32x4*>(a.col_max + m_first + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) up[e] = power_of(up_of(bits[e]));
          }
        }
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
        for (int j = 0; j < kT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * q + e;
            *reinterpret_cast<uint16_t*>(own + r * kRow + (((2 * j + (row >> 3)) ^ (r % kCh)) << 4) +
                                         2 * (row & 7)) = (uint16_t)T::pack(acc[i][j][e] * up[e], 0.f);
          }
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
        for (int s = 0; s < (16 + kPer - 1) / kPer; ++s) {
          const int r = s * kPer + lane / kCh, c = (lane % kCh) ^ (r % kCh), m = m_first + r;
          if (kPer > 16 && r >= 16) continue;
          const u32x4 v = *reinterpret_cast<const u32x4*>(own + r * kRow + (lane % kCh) * 16);
          if (m < a.f && tw + 8 * c < a.np)
            *reinterpret_cast<u32x4*>(a.dt + ((int64_t)(i < kH ? 0 : a.f) + m) * a.np + tw + 8 * c) = v;
        }
      }
    }
  }
}

template <class T, class A, class P, int G, bool GRAD>
__global__ __launch_bounds__(G * P::kThreads, 1) void gated_kernel(GatedArgs a) {
  gated_tile<T, A, P, G, GRAD>(a);
}

// Up to 32 rows by 16 columns of h per workgroup.  Four waves split k and sum in LDS; two workgroups a CU, so that one's
// loads are on their way while the other starts or ends, and the weights, which the call reads once, go past the
// caches.  Bound by the weights: 235 MB of 4096 -> 14336 (out of the caches) 1 row 38 us, 6.2 TB/s, 32 rows 45 us (eight
// waves, one workgroup a CU: 46 and 53; through the caches 42 and 49).
constexpr int kFewWaves = 8, kGatedWaves = 4;
template <class T>
using GatedFew = WaveProduct<T, 1, 1, 2, 32, true, true>;
template <class T>
constexpr int kGatedFewLds = kGatedWaves * GatedFew<T>::kBytes;

template <class T, class A, bool GRAD>
__device__ __forceinline__ void gated_few(const GatedArgs& a) {
  using P = GatedFew<T>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = (int)blockIdx.x * 16;
  const int nk = (a.k + 63) / 64;
  f32x16 acc[1][1];
  unsigned char* own = smem + wave * P::kBytes;
  const int64_t w0 = (int64_t)m0 * a.k;
  P::run(a.x, (int)a.x_ld, (int)a.n - 1,
         {{a.wg + w0, a.wu + w0}, a.k, a.f - m0 < 16 ? a.f - m0 - 1 : 15}, a.k, nk * wave / kGatedWaves,
         nk * (wave + 1) / kGatedWaves, own, lane, acc);
  float* part = reinterpret_cast<float*>(own);  // [16][64]
#pragma unroll
  for (int r = 0; r < 16; ++r) part[r * 64 + lane] = acc[0][0][r];
  __syncthreads();
  // thread: two columns of a row.  Column m < 16 of wg is entry e = 4 (m / 8) + m % 4 of lane
  // (row, half (m / 4) % 2), that of wu entry e + 8.
  const int row = threadIdx.x & 31, m = 2 * (threadIdx.x >> 5);
  const int e = 4 * (m >> 3) + (m & 3), from = row + 32 * ((m >> 2) & 1);
  float g[2] = {0.f, 0.f}, u[2] = {0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kGatedWaves; ++w) {
    const float* p = reinterpret_cast<const float*>(smem + w * P::kBytes) + from;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      g[c] += p[(e + c) * 64];
      u[c] += p[(e + 8 + c) * 64];
    }
  }
  const int64_t t = row;
  if (m0 + m >= a.f) return;
  if constexpr (!GRAD) {
    if (t < a.n)
      *reinterpret_cast<uint32_t*>(a.h + t * a.f + m0 + m) =
          T::pack(A::value(g[0]) * u[0], A::value(g[1]) * u[1]);
  } else {
    float dg[2] = {0.f, 0.f}, du[2] = {0.f, 0.f};
    if (t < a.n) {
      const uint32_t b = *reinterpret_cast<const uint32_t*>(a.dh + t * a.f + m0 + m);
      gradients<A>(g[0], u[0], T::lo(b), dg[0], du[0]);
      gradients<A>(g[1], u[1], T::hi(b), dg[1], du[1]);
      if (a.d) {
        float up = 1.f;
        if constexpr (T::kNarrow) up = power_of(up_of(a.row_max[t]));
        uint16_t* d = a.d + t * 2 * a.f + m0 + m;
        *reinterpret_cast<uint32_t*>(d) = T::pack(dg[0] * up, dg[1] * up);
        *reinterpret_cast<uint32_t*>(d + a.f) = T::pack(du[0] * up, du[1] * up);
      }
    }
    if (a.dt && t < a.np) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float up = 1.f;
        if constexpr (T::kNarrow) up = power_of(up_of(a.col_max[m0 + m + c]));
        uint16_t* d = a.dt + (int64_t)(m0 + m + c) * a.np + t;
        d[0] = (uint16_t)T::pack(dg[c] * up, 0.f);
        d[(int64_t)a.f * a.np] = (uint16_t)T::pack(du[c] * up, 0.f);
      }
    }
  }
}

template <class T, class A, bool GRAD>
__global__ __launch_bounds__(64 * kGatedWaves) void gated_few_kernel(GatedArgs a) {
  static_assert(kGatedWaves == 4, "a thread for every two columns of 32 rows");
  gated_few<T, A, GRAD>(a);
}

// ---- dx, dW -------------------------------------------------------------------------------------

// y[r][c] = 2^-up(r) <x_r, w_c>, rows [0, split) to y[0], the others to y[1].  Where the tiles are too few for the chip and
// k is long, `splits` workgroups share a tile's k, and their sums go to memory in 32 bits for join_kernel.
template <class T, class P, int G>
__device__ __forceinline__ void rows_tile(const ProductArgs& a) {
  constexpr int kT = P::kT, kM = P::kM;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // P::kLds
  const int lane = threadIdx.x & 63, row = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wave % P::kWt, wm = wave % P::kW / P::kWt;  // (of group 0, which stores)
  const int n_m = (a.m + P::kCols - 1) / P::kCols;
  const uint32_t n_t = (uint32_t)((a.n - a.row0 + P::kRows - 1) / P::kRows);
  // (an XCD's workgroups are tiles of the same part of k, and share its lines)
  const uint32_t lin = (uint32_t)xcd_linear(blockIdx.x, gridDim.x), part = lin / (n_t * (uint32_t)n_m);
  const TileAt at = tile_of(lin - part * n_t * n_m, n_t, n_m);
  const int each = ((a.k + 63) / 64 + a.splits - 1) / a.splits * 64, k0 = (int)part * each;
  const int left_k = a.k - k0 < each ? a.k - k0 : each;
  const int64_t t0 = a.row0 + (int64_t)at.t * P::kRows;
  const int m0 = at.m * P::kCols;
  const int64_t left_t = a.n - t0;
  const int last_t = left_t < P::kRows ? (int)left_t - 1 : P::kRows - 1;
  const int last_m = a.m - m0 < P::kCols ? a.m - m0 - 1 : P::kCols - 1;
  typename P::Acc acc;
  const uint16_t* const w0 = a.w + (int64_t)m0 * a.ld + k0;
  if (!grouped<P, G>(a.x + t0 * a.ld + k0, a.ld, last_t, {{w0, w0}, a.ld, last_m}, left_k > 0 ? left_k : 0, at, smem,
                     wave, lane, acc))
    return;
  constexpr int kOwn = 16 * 32 * kM, kSums = (G - 1) * P::kW * kM * kT * 1024;
  static_assert(kSums + P::kW * kOwn <= G * P::kLds, "the waves' blocks fit beside the sums");
  unsigned char* own = smem + kSums + wave * kOwn;
  const int mw = m0 + wm * P::kWaveCols;
  if (a.splits > 1) {
#pragma unroll
    for (int j = 0; j < kT; ++j) {
      const int64_t r = t0 + (wt * kT + j) * 16 + row;
      float* to = a.part + ((int64_t)part * a.n + r) * a.m + mw + 4 * (lane >> 4);
#pragma unroll
      for (int i = 0; i < kM; ++i)
        if (r < a.n && mw + 16 * i + 4 * (lane >> 4) < a.m) *reinterpret_cast<f32x4*>(to + 16 * i) = acc[i][j];
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kT; ++j) {
    const int64_t r0 = t0 + (wt * kT + j) * 16;
    float down = 1.f;
    if constexpr (T::kNarrow) {
      const int64_t t = r0 + row < a.n ? r0 + row : a.n - 1;
      down = power_of(-up_of(a.max_bits[t < a.split ? t : t - a.split]));
    }
    auto value = [&](int i, int e) { return acc[i][j][e] * down; };
    // (the split may lie inside a tile: every row goes to the output that it is of)
    const int64_t n_first = a.n < a.split ? a.n : a.split;
    if (r0 < a.split) store_rows16<T, kM>(a.y[0] + r0 * a.m + mw, a.m, n_first - r0, a.m - mw, own, lane, value);
    if (r0 + 16 > a.split && a.n > a.split)
      store_rows16<T, kM>(a.y[1] + (r0 - a.split) * a.m + mw, a.m, a.n - r0, a.m - mw, own, lane, value,
                          a.split - r0);
  }
}

template <class T, class P, int G>
__global__ __launch_bounds__(G * P::kThreads, 1) void rows_kernel(ProductArgs a) {
  rows_tile<T, P, G>(a);
}

// The splits' sums, in their order: eight values a thread.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, all = a.n * a.m;
  if (i >= all) return;
  f32x4 v[2] = {};
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    const f32x4* from = reinterpret_cast<const f32x4*>(a.part + s * all + i);
    v[0] += from[0];
    v[1] += from[1];
  }
  const int64_t t = i / a.m, c = i - t * a.m;
  const bool first = t < a.split;
  const int64_t at = first ? t : t - a.split;
  float down = 1.f;
  if constexpr (T::kNarrow) down = power_of(-up_of(a.max_bits[at]));
  u32x4 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) w[q] = T::pack(v[q >> 1][2 * (q & 1)] * down, v[q >> 1][2 * (q & 1) + 1] * down);
  *reinterpret_cast<u32x4*>(a.y[first ? 0 : 1] + at * a.m + c) = w;
}

// Few tiles: 32 rows by 32 columns, eight waves split k.
template <class T>
using RowsFew = WaveProduct<T, 1, 1>;
template <class T>
constexpr int kRowsFewLds = kFewWaves * RowsFew<T>::kBytes;

template <class T>
__device__ __forceinline__ void rows_few(const ProductArgs& a) {
  using P = RowsFew<T>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t n_m = (uint32_t)(a.m + 31) / 32u;
  const int m0 = (int)(blockIdx.x % n_m) * 32;
  const int64_t t0 = (int64_t)(blockIdx.x / n_m) * 32;
  const int nk = (a.k + 63) / 64;
  f32x16 acc[1][1];
  unsigned char* own = smem + wave * P::kBytes;
  P::run(a.x + t0 * a.ld, a.ld, a.n - t0 < 32 ? (int)(a.n - t0) - 1 : 31,
         {{a.w + (int64_t)m0 * a.ld, nullptr}, a.ld, a.m - m0 < 32 ? a.m - m0 - 1 : 31}, a.k,
         nk * wave / kFewWaves, nk * (wave + 1) / kFewWaves, own, lane, acc);
  float* part = reinterpret_cast<float*>(own);  // [16][64]
#pragma unroll
  for (int r = 0; r < 16; ++r) part[r * 64 + lane] = acc[0][0][r];
  __syncthreads();
  // thread: two columns of a row; column m < 32 is entry 4 (m / 8) + m % 4 of lane (row, half (m / 4) % 2)
  const int row = threadIdx.x & 31, m = 2 * (threadIdx.x >> 5);
  const int e = 4 * (m >> 3) + (m & 3), from = row + 32 * ((m >> 2) & 1);
  float v[2] = {0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    const float* p = reinterpret_cast<const float*>(smem + w * P::kBytes) + from;
    v[0] += p[e * 64];
    v[1] += p[(e + 1) * 64];
  }
  const int64_t t = t0 + row;
  if (t >= a.n || m0 + m >= a.m) return;
  const bool first = t < a.split;
  const int64_t at = first ? t : t - a.split;
  float down = 1.f;
  if constexpr (T::kNarrow) down = power_of(-up_of(a.max_bits[at]));
  *reinterpret_cast<uint32_t*>(a.y[first ? 0 : 1] + at * a.m + m0 + m) = T::pack(v[0] * down, v[1] * down);
}

template <class T>
__global__ __launch_bounds__(64 * kFewWaves) void rows_few_kernel(ProductArgs a) {
  rows_few<T>(a);
}

// dx of few rows, from the weights as they lie: dx[t][c] = sum_j d[t][j] w[j][c], where the weights' rows j are read in
// tiles of 64 rows by 64 columns and their columns taken by the LDS reads (tr_frag), so that nothing is transposed
// first.  A workgroup takes 32 TB rows by 64 columns and a part of the sum, its four waves a quarter of it each, without a
// barrier; they join in LDS and the parts in join_kernel.  Bound by the weights, which are read once for every 32 TB
// rows: x's gradients of 64 rows, 4096 -> 14336, d's product included: 104 us, with the weights transposed first 224.
template <int TB>
constexpr int kColumnsStages = TB == 1 ? 3 : 2;
template <int TB>
constexpr int kColumnsStage = 8192 + TB * 4096;  // bytes: 64 rows of w's 64 columns, 32 TB rows of d's 64 values
constexpr int kColumnsWaves = 4;
template <int TB>
constexpr int kColumnsLds = kColumnsWaves * kColumnsStages<TB> * kColumnsStage<TB>;

template <class T, int TB>
__device__ __forceinline__ void columns_few(const ColumnsArgs& a) {
  constexpr int kStages = kColumnsStages<TB>, kStage = kColumnsStage<TB>, kLoads = 8 + 4 * TB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // kColumnsLds
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t n_c = (uint32_t)(a.k + 63) / 64u, n_t = (uint32_t)((a.n + 32 * TB - 1) / (32 * TB));
  const int c0 = (int)(blockIdx.x % n_c) * 64;
  const int64_t t0 = (int64_t)(blockIdx.x / n_c % n_t) * 32 * TB;
  const int part = (int)(blockIdx.x / n_c / n_t);
  // stages of wg's rows, then of wu's; this wave's are [s0, s1)
  const int of_one = (a.f + 63) / 64, unit = part * kColumnsWaves + wave, units = a.splits * kColumnsWaves;
  const int s0 = (int)((int64_t)2 * of_one * unit / units), s1 = (int)((int64_t)2 * of_one * (unit + 1) / units);
  const int64_t left_t = a.n - t0;
  const int last_t = left_t < 32 * TB ? (int)left_t - 1 : 32 * TB - 1;
  const int last_c = a.k - c0 < 64 ? a.k - c0 - 8 : 56;
  unsigned char* const own = smem + wave * kStages * kStage;
  const uint32_t lds = LDS_ADDRESS(smem) + wave * kStages * kStage;
  const int lr = lane >> 3;  // row of a wave load, 8 rows of 8 chunks
  // (a row of w past the last repeats it: d is zero there)
  auto issue = [&](int buf, int s) __attribute__((always_inline)) {
    const bool up = s >= of_one;
    const int f0 = (up ? s - of_one : s) * 64, n_f = a.f - f0 < 64 ? a.f - f0 : 64;
    const rsrc_t rw = rsrc_of((up ? a.wu : a.wg) + (int64_t)f0 * a.k + c0);
    const uint16_t* const d = a.d + t0 * 2 * a.f + (up ? a.f : 0) + f0;
    const uint32_t st = lds + buf * kStage;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 8 * j + lr, c = 8 * ((lane & 7) ^ swz<64>(r)), in = r < n_f ? r : n_f - 1;
      load_lds16_stream(rw, st + j * 1024, (uint32_t)(in * a.k + (c < last_c ? c : last_c)) * 2u);
    }
#pragma unroll
    for (int j = 0; j < 4 * TB; ++j) {
      const int r = 8 * j + lr, c = 8 * ((lane & 7) ^ swz<64>(r));
      const uint16_t* from = d + (int64_t)(r < last_t ? r : last_t) * 2 * a.f + c;
      load_lds16(c < n_f ? (const void*)from : (const void*)kZero16, st + 8192 + j * 1024);
    }
  };
  f32x16 acc[2][TB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const TileReads<64> rd(lane);
#pragma unroll
  for (int q = 0; q < kStages - 1; ++q)
    if (s0 + q < s1) issue(q, s0 + q);
#pragma unroll 1
  for (int s = s0, buf = 0; s < s1; ++s, buf = buf + 1 < kStages ? buf + 1 : 0) {
    if (s + kStages - 1 < s1) {
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);  // that stage's reads are done
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      issue(buf > 0 ? buf - 1 : kStages - 1, s + kStages - 1);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm((kStages - 1) * kLoads));
    } else if (kStages == 3 && s + 1 < s1) {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(kLoads));
    } else {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    }
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    const unsigned char* ws = own + buf * kStage;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        // d's values in tr_frag's order of rows: 8 (e / 4) + 4 half + e % 4 of these 16
        u32x4 fd[TB];
#pragma unroll
        for (int j = 0; j < TB; ++j) {
          const int r = 32 * j + col, c = 4 * b + 2 * st;
          const unsigned char* row = ws + 8192 + r * 128 + 8 * half;
          const uint2 lo = *reinterpret_cast<const uint2*>(row + ((c ^ swz<64>(r)) << 4));
          const uint2 hi = *reinterpret_cast<const uint2*>(row + (((c + 1) ^ swz<64>(r)) << 4));
          fd[j] = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x4 fw = rd.tr_frag(ws, b, st, i);
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[i][j] = T::mfma(fw, fd[j], acc[i][j]);
        }
      }
  }
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  float* const sums = reinterpret_cast<float*>(own);  // [2 TB * 16][64]
  static_assert(2 * TB * 4096 <= kStages * kStage, "the wave's sums fit its stages");
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums[(16 * (i * TB + j) + r) * 64 + lane] = acc[i][j][r];
  __syncthreads();
  // four columns of a row at a time: entries 4 g .. 4 g + 3 of block (i, j)
  for (int q = wave; q < 8 * TB; q += kColumnsWaves) {
    const int g = q & 3, i = (q >> 2) / TB, j = (q >> 2) % TB;
    const int c = c0 + 32 * i + 8 * g + 4 * half;
    const int64_t t = t0 + 32 * j + col;
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kColumnsWaves; ++w)
        v[e] += reinterpret_cast<const float*>(smem + w * kStages * kStage)[(4 * q + e) * 64 + lane];
    }
    if (t < a.n && c < a.k) *reinterpret_cast<f32x4*>(a.part + ((int64_t)part * a.n + t) * a.k + c) = v;
  }
}

template <class T, int TB>
__global__ __launch_bounds__(64 * kColumnsWaves) void columns_kernel(ColumnsArgs a) {
  columns_few<T, TB>(a);
}

// ---- transposes ---------------------------------------------------------------------------------

// Up to three matrices [rows, cols] (multiples of 8 columns) in one launch, a 64 x 64 tile per workgroup:
// out[c][r] (rows of `ld`, zero from `rows` to the next multiple of 8), of 16-bit values or of a checkpoint's
// codes, whose values then go to `plain` as well.  And clears `words` for max_kernel.
template <class T>
__global__ __launch_bounds__(256) void prepare_kernel(GatedPrepare a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[64][72];
  uint32_t b = blockIdx.x;
  if (b < a.clear_blocks) {
    const int64_t i = (int64_t)b * 256 + threadIdx.x;
    if (i < a.words) a.clear[i] = 0;
    return;
  }
  b -= a.clear_blocks;
  int w = 0;
  while (w < 2 && b >= a.job[w].blocks) b -= a.job[w++].blocks;
  const GatedTranspose& q = a.job[w];
  const uint32_t n_c = (uint32_t)(q.cols + 63) / 64u;
  const int64_t r0 = (int64_t)(b / n_c) * 64;
  const int c0 = (int)(b % n_c) * 64;
  const int x = 8 * (threadIdx.x & 7), y = threadIdx.x >> 3;
#pragma unroll
  for (int i = y; i < 64; i += 32) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (r0 + i < q.rows && c0 + x < q.cols) {
      if (q.codes) {
        v = unpack8<T>(*reinterpret_cast<const uint2*>(q.codes + (r0 + i) * q.cols + c0 + x),
                       q.exps[(r0 + i) * ((q.cols + 31) / 32) + (c0 + x) / 32]);
        if (q.plain) *reinterpret_cast<u32x4*>(q.plain + (r0 + i) * q.cols + c0 + x) = v;
      } else {
        v = load16(q.in + (r0 + i) * q.in_ld + c0 + x);
      }
    }
    *reinterpret_cast<u32x4*>(&tile[i][x]) = v;
  }
  if (!q.out) return;
  __syncthreads();
  // thread: 8 rows of one column; a wave's 64 columns of the same rows read LDS without conflicts
  const int c = threadIdx.x & 63;
#pragma unroll
  for (int k = threadIdx.x >> 6; k < 8; k += 4) {
    if (c0 + c >= q.cols || r0 + 8 * k >= q.rows) continue;
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = (uint32_t)tile[8 * k + 2 * e][c] | (uint32_t)tile[8 * k + 2 * e + 1][c] << 16;
    *reinterpret_cast<u32x4*>(q.out + (int64_t)(c0 + c) * q.ld + r0 + 8 * k) = v;
  }
}

// ---- launches -----------------------------------------------------------------------------------

// Tiles of rows by rows of the weights (of a paired tile half of them of each matrix).
template <class T, bool PAIR>
using Wide = TileProduct16<T, 256, 256, 4, 2, 3, 2, PAIR>;
template <class T, bool PAIR>
using Middle = TileProduct16<T, 128, 128, 4, 2, 4, 4, PAIR>;
template <class T, bool PAIR>
using Small = TileProduct16<T, 64, 64, 2, 2, 3, 2, PAIR>;
constexpr int kSmallGroups = 4;  // of its waves, which split k

// The dynamic LDS of a kernel beyond the default limit.
hipError_t allow_lds(const void* fn, int lds) {
  return lds > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds) : hipSuccess;
}

template <class T, class A, class P, bool GRAD, int G = 1>
hipError_t gated_as(const GatedArgs& a, hipStream_t s) {
  const int64_t grid = (a.n + P::kRows - 1) / P::kRows * ((a.f + P::kCols - 1) / P::kCols);
  const auto kernel = gated_kernel<T, A, P, G, GRAD>;
  const hipError_t e = allow_lds((const void*)kernel, G * P::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(G * P::kThreads), G * P::kLds, s, a);
  return hipGetLastError();
}

template <class T, class A, bool GRAD>
hipError_t gated_few_as(const GatedArgs& a, hipStream_t s) {
  constexpr int lds = kGatedFewLds<T>;
  const auto kernel = gated_few_kernel<T, A, GRAD>;
  const hipError_t e = allow_lds((const void*)kernel, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.f + 15) / 16u), dim3(64 * kGatedWaves), lds, s, a);
  return hipGetLastError();
}

// The tile of h, or of d, by the number of tiles (h alone, us; rows, k -> f):
//   one row of tiles of 16 columns   up to 32 rows
//   64 x 32     up to 256 of these: 146 rows, 768 -> 2304 (216 tiles) 6.8 (128 x 64: 8.2), 96 rows, 4096 -> 4096 (256) 17.5
//               (26.5); 200 rows, 768 -> 2304 (288) 11.0 (8.1), 48 rows, 4096 -> 14336 (448) 39 (36)
//   128 x 64    otherwise, until
//   256 x 128   there are 144 of these: 1,500 rows, 768 -> 2304 (108) 19.6 (16.2), 2,048 rows (144) 20.8 (23.9), 1,024 rows,
//               4096 -> 4096 (128) 78 (65), 1,500 rows (192) 84 (95)
template <class T, class A, bool GRAD>
hipError_t gated(const GatedArgs& a, hipStream_t s) {
  auto tiles = [&](int t, int m) { return (a.n + t - 1) / t * ((a.f + m - 1) / m); };
  if (a.n <= 32) return gated_few_as<T, A, GRAD>(a, s);
  if (tiles(64, 32) <= 256) return gated_as<T, A, Small<T, true>, GRAD, kSmallGroups>(a, s);
  if (tiles(256, 128) >= 144) return gated_as<T, A, Wide<T, true>, GRAD>(a, s);
  return gated_as<T, A, Middle<T, true>, GRAD>(a, s);
}

template <class T, bool GRAD>
hipError_t gated_act(const GatedArgs& a, hipStream_t s) {
  switch (a.act) {
    case 0: return gated<T, Silu, GRAD>(a, s);
    case 1: return gated<T, Gelu, GRAD>(a, s);
    default: return gated<T, GeluTanh, GRAD>(a, s);
  }
}

template <class T, class P, int G = 1>
hipError_t rows_as(const ProductArgs& a, hipStream_t s) {
  const int64_t grid = (a.n - a.row0 + P::kRows - 1) / P::kRows * ((a.m + P::kCols - 1) / P::kCols) * a.splits;
  const auto kernel = rows_kernel<T, P, G>;
  const hipError_t e = allow_lds((const void*)kernel, G * P::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(G * P::kThreads), G * P::kLds, s, a);
  return hipGetLastError();
}

// How a product's tiles are made: the least estimated time, of 256 workgroups at a time, a stage of 64 values of k taking
// a tile what it took in calls of 1 to 1,000 rows (256 x 256 1.26 us, 128 x 128 0.55, 64 x 64 by four groups of waves 0.29,
// 32 x 32 by eight waves 0.14), and the splits' sums 8 bytes a value, written and read at 3.5 TB/s, and a launch.
// The gradients of x alone, us with splits (without): 764 rows, 4096 -> 14336 (k 28672) 476 (578), 300 rows 331 (493),
// 1,500 rows 738 (936), 764 rows, 768 -> 2304 (k 4608) 35 (39), 450 rows, 1024 -> 4096 45 (54).
struct RowsPlan {
  int tile;  // 0: 32 x 32, 1: 64 x 64, 2: 128 x 128, 3: 256 x 256
  int splits;
};
RowsPlan rows_plan(int64_t n, int m, int k) {
  constexpr int kSize[4] = {32, 64, 128, 256};
  constexpr int kThreads[4] = {64 * kFewWaves, kSmallGroups * Small<HalfBf16, false>::kThreads,
                               Middle<HalfBf16, false>::kThreads, Wide<HalfBf16, false>::kThreads};
  constexpr double kStage[4] = {0.143, 0.29, 0.55, 1.26};
  const int64_t stages = k > 0 ? (k + 63) / 64 : 1;
  RowsPlan best = {3, 1};
  double least = 0.0;
  for (int t = 3; t >= 0; --t) {
    const int64_t tiles = (n + kSize[t] - 1) / kSize[t] * ((m + kSize[t] - 1) / kSize[t]);
    if (t < 3 && !launch_fits(tiles, kThreads[t])) continue;  // (gated_fits has asked for those of 256)
    const int most = t < 2 || tiles >= 256 ? 1 : 16;
    for (int s = 1; s <= most && (s == 1 || (tiles * s <= 256 && stages / s >= 4)); ++s) {
      const double rounds = (double)((tiles * s + 255) / 256), part = (double)((stages + s - 1) / s);
      const double us = rounds * part * kStage[t] + (s > 1 ? 8.0 + (double)s * (double)n * m * 8.0 / 3.5e6 : 0.0);
      if (t == 3 && s == 1) least = us;
      if (us < least) {
        least = us;
        best = {t, s};
      }
    }
  }
  return best;
}

template <class T>
hipError_t rows(ProductArgs a, hipStream_t s) {
  const RowsPlan plan = rows_plan(a.n, a.m, a.k);
  a.splits = plan.splits;
  hipError_t e = hipSuccess;
  if (plan.tile == 0) {
    const auto kernel = rows_few_kernel<T>;
    e = allow_lds((const void*)kernel, kRowsFewLds<T>);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.n + 31) / 32 * ((a.m + 31) / 32))), dim3(64 * kFewWaves),
                       kRowsFewLds<T>, s, a);
    return hipGetLastError();
  }
  if (plan.tile == 1) return rows_as<T, Small<T, false>, kSmallGroups>(a, s);
  if (plan.tile == 2) {
    e = rows_as<T, Middle<T, false>>(a, s);
  } else {
    // a last round of up to 112 tiles (of 256, one a CU) is left to the next size
    const int64_t n_m = (a.m + 255) / 256, tiles = (a.n + 255) / 256 * n_m, rest = tiles % 256;
    const int64_t whole = (tiles - rest) / n_m * 256;  // rows of the whole rounds
    ProductArgs w = a;
    if (a.splits == 1 && rest > 0 && rest <= 112 && whole > 0) w.n = whole;
    e = rows_as<T, Wide<T, false>>(w, s);
    if (e == hipSuccess && w.n < a.n) {
      a.row0 = whole;
      e = rows_as<T, Middle<T, false>>(a, s);
    }
  }
  if (e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)((a.n * a.m / 8 + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class T, int TB>
hipError_t columns_as(const ColumnsArgs& a, hipStream_t s) {
  const auto kernel = columns_kernel<T, TB>;
  const hipError_t e = allow_lds((const void*)kernel, kColumnsLds<TB>);
  if (e != hipSuccess) return e;
  const int64_t grid = (a.k + 63) / 64 * ((a.n + 32 * TB - 1) / (32 * TB)) * a.splits;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kColumnsWaves), kColumnsLds<TB>, s, a);
  return hipGetLastError();
}

// Parts of the sum: two rounds of workgroups, of two stages a wave at least.
int columns_splits(int64_t n, int k, int f) {
  const int64_t tiles = (k + 63) / 64 * (n <= 32 ? 1 : (n + 63) / 64);
  int64_t s = 512 / tiles;
  const int64_t most = (f + 63) / 64 * 2 / (2 * kColumnsWaves);
  s = s < most ? s : most;
  return s < 1 ? 1 : (int)s;
}

template <class T>
hipError_t columns(ColumnsArgs a, uint16_t* dx, const uint32_t* row_max, hipStream_t s) {
  a.splits = columns_splits(a.n, a.k, a.f);
  const hipError_t e = a.n <= 32 ? columns_as<T, 1>(a, s) : columns_as<T, 2>(a, s);
  if (e != hipSuccess) return e;
  ProductArgs q = {nullptr, nullptr, a.n, a.k, 0, 0, {dx, nullptr}, a.n, row_max, a.part};
  q.splits = a.splits;
  hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)((a.n * a.k / 8 + 255) / 256)), dim3(256), 0, s, q);
  return hipGetLastError();
}

}  // namespace

// dx by columns_kernel up to here, from transposed weights past it (us, 4096 -> 14336 and 768 -> 2304): 160 rows 224 and
// 24.6 (transposed 276 and 25.0), 192 rows 226 and 25.8 (280 and 25.4), 256 rows 266 and 30.6 (290 and 28.5).
bool gated_by_columns(int64_t n) { return n <= 192; }

size_t gated_columns_bytes(int64_t n, int k, int f) {
  return (size_t)columns_splits(n, k, f) * n * k * sizeof(float);
}

hipError_t launch_gated_columns(const ColumnsArgs& a, bool f16, uint16_t* dx, const uint32_t* row_max,
                                hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  return f16 ? columns<HalfF16>(a, dx, row_max, stream) : columns<HalfBf16>(a, dx, row_max, stream);
}

// (Where a limit is near, the tiles are 256 x 128 and 256 x 256 by 512 threads, and max_kernel's of 64 rows; rows_plan
// leaves out smaller ones that do not fit.)
bool gated_fits(int64_t n, int k, int f, bool grads) {
  auto blocks = [](int64_t size, int of) { return (size + of - 1) / of; };
  if (!launch_fits(blocks(n, 256) * blocks(f, 128), 512)) return false;
  if (!grads) return true;
  const int64_t prepare = blocks(n + f, 256) + 2 * blocks(f, 64) * blocks(k, 64) + blocks(n, 64) * blocks(k, 64);
  return launch_fits(prepare, 256) && launch_fits(blocks(n, 64) * blocks(f, 512), 256) &&
         launch_fits(blocks(n, 256) * blocks(k, 256), 512);
}

hipError_t launch_gated(const GatedArgs& a, bool grad, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  if (grad) return a.f16 ? gated_act<HalfF16, true>(a, stream) : gated_act<HalfBf16, true>(a, stream);
  return a.f16 ? gated_act<HalfF16, false>(a, stream) : gated_act<HalfBf16, false>(a, stream);
}

size_t rows_product_bytes(int64_t n, int m, int k) {
  const int splits = rows_plan(n, m, k).splits;
  return splits > 1 ? (size_t)splits * n * m * sizeof(float) : 0;
}

hipError_t launch_rows_product(const ProductArgs& a, bool f16, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  return f16 ? rows<HalfF16>(a, stream) : rows<HalfBf16>(a, stream);
}

hipError_t launch_gated_max(const uint16_t* dh, int64_t n, int f, uint32_t* rows, uint32_t* cols,
                            hipStream_t stream) {
  if (n == 0) return hipSuccess;
  // fewer atomics where there are workgroups enough
  const int64_t n_c = (f + 511) / 512;
  if ((n + 63) / 64 * n_c >= 1024)
    hipLaunchKernelGGL(max_kernel<16>, dim3((unsigned)((n + 63) / 64 * n_c)), dim3(256), 0, stream, dh, n, f, rows, cols);
  else
    hipLaunchKernelGGL(max_kernel<4>, dim3((unsigned)((n + 15) / 16 * n_c)), dim3(256), 0, stream, dh, n, f, rows, cols);
  return hipGetLastError();
}

hipError_t launch_gated_prepare(GatedPrepare a, bool f16, hipStream_t stream) {
  a.clear_blocks = (uint32_t)((a.words + 255) / 256);
  int64_t blocks = a.clear_blocks;
  for (GatedTranspose& q : a.job) {
    q.blocks = (uint32_t)((q.rows + 63) / 64 * ((q.cols + 63) / 64));
    blocks += q.blocks;
  }
  if (blocks == 0) return hipSuccess;
  if (f16)
    hipLaunchKernelGGL(prepare_kernel<HalfF16>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(prepare_kernel<HalfBf16>, dim3((unsigned)blocks), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace hpr
