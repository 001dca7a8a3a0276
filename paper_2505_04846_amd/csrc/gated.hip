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
// with the weights' columns, and dW one of d's columns with x's: d is written both ways round by the epilogue, the
// weights' and x's columns are taken by the LDS reads.
#include "checkpoint.h"
#include "common.h"
#include "half.h"
#include "kernels.h"
#include "product.h"
#include "tiles.h"

namespace hpr {

namespace {

// ---- activations ------------------------------------------------------------------------------

// exp of a 32-bit number, relative error (1.25 |x| + 2) 2^-24 (the product's rounding, the constant's, 0.22 2^-24, and
// the instruction's): far below the rounding of what it goes into.
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

// dg and du are products' operands in 16 bits, rounded once.  That makes dx and dW 1.4 times as far off as outputs' own
// rounding alone would (bf16 2.3e-3 of their norm beside 1.7e-3, fp16 2.9e-4 beside 2.1e-4); in two numbers each they
// would double the products of dx and dW, half of the time of all gradients.
// fp16 has few exponents: where dh is small (a loss that is not scaled), they would lose bits below 2^-14.  So a row of
// d is written for dx times the power of two that brings the row's largest |dh| into [1/4, 1/2), a column for dW times
// that of its column, and the products' results are multiplied back in 32 bits: exactly undone, whatever the size of
// dh.  What is left are the factors act(g) and u act'(g).  Where g and u are numbers of fp16 these are at most 1.13 times
// 65504, and half of that is a number of fp16 too; a larger power would not do, finite as h may be (g of 0.5 and u of
// 60,000: h of 18,700, u act'(g) of 44,400, which [1, 2) makes infinite).  They overflow from 131,040 on, which g or u
// passes 65504 for, and lose bits below 2^-12 (h, as a number of fp16, does below 2^-14).
// bits: the largest |value| of fp16 as a whole number (max_kernel); 0 and infinities stay as they are.
__device__ __forceinline__ int up_of(uint32_t bits) {
  if (bits == 0 || bits >= 0x7c00) return 0;
  const float v = (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
  return 125 - (int)(__float_as_uint(v) >> 23);
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
constexpr int kGatedWaves = 4;
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

// y[r][c] = 2^-up(r) sum_j x[r][j] w[j][c], rows [0, split) to y[0], the others to y[1]: dx of d and the weights, dW of d
// transposed and x, whose columns the LDS reads take (PanelT in product.h), so that neither is transposed first (us, with
// both transposed and smaller tiles beside these: all gradients of 6,529 rows, 4096 -> 14336 3,787, now 3,647, of 764 rows
// 658 and 549, 764 rows, 768 -> 2304 49 and 42; 1 row, 4096 -> 14336, in a kernel of its own that streamed the weights past
// the caches, 143 and 166).  Bound by the matrix cores' power limit in large calls, by the weights in small ones.  Where
// the tiles are too few for the chip and k is long, `splits` workgroups share a tile's k, and their sums go to memory in
// 32 bits for join_kernel.
template <class T, class P>
__device__ __forceinline__ void rows_tile(const ProductArgs& a) {
  constexpr int kT = P::kT, kM = P::kM;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // P::kLds
  const int lane = threadIdx.x & 63, row = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wave % P::kWt, wm = wave / P::kWt;
  const int n_m = (a.m + P::kCols - 1) / P::kCols;
  const uint32_t n_t = (uint32_t)((a.n - a.row0 + P::kRows - 1) / P::kRows);
  // (an XCD's workgroups are tiles of the same part of k, and share its lines)
  const uint32_t lin = (uint32_t)xcd_linear(blockIdx.x, gridDim.x), part = lin / (n_t * (uint32_t)n_m);
  const TileAt at = tile_of(lin - part * n_t * n_m, n_t, n_m);
  const int each = ((a.k + 63) / 64 + a.splits - 1) / a.splits * 64, k0 = (int)part * each;
  const int left_k = k0 >= a.k ? 0 : a.k - k0 < each ? a.k - k0 : each;
  const int64_t t0 = a.row0 + (int64_t)at.t * P::kRows;
  const int m0 = at.m * P::kCols;
  const int64_t left_t = a.n - t0;
  const int last_t = left_t < P::kRows ? (int)left_t - 1 : P::kRows - 1;
  const int last_m = a.m - m0 < P::kCols ? a.m - m0 - 1 : P::kCols - 1;
  typename P::Acc acc;
  P::run(a.x + t0 * a.ld + k0, a.ld, last_t, PanelT{{a.w[0] + m0, a.w[1] + m0}, a.w_ld, last_m, k0, a.half}, left_k,
         (left_k + 63) / 64, at, smem, wave, lane, acc);
  constexpr int kOwn = 16 * 32 * kM;
  static_assert(P::kW * kOwn <= P::kLds, "the waves' blocks fit");
  unsigned char* own = smem + wave * kOwn;
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

template <class T, class P>
__global__ __launch_bounds__(P::kThreads, 1) void rows_kernel(ProductArgs a) {
  rows_tile<T, P>(a);
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

// Words to zero (a kernel, which a captured graph replays as it was).
__global__ __launch_bounds__(256) void clear_kernel(uint32_t* words, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) words[i] = 0;
}

// ---- launches -----------------------------------------------------------------------------------

// Tiles of rows by rows of the weights (of a paired tile half of them of each matrix).
template <class T, bool PAIR>
using Wide = TileProduct16<T, 256, 256, 4, 2, 3, 2, PAIR>;
template <class T, bool PAIR>
using Middle = TileProduct16<T, 128, 128, 4, 2, 4, 4, PAIR>;
template <class T>
using Small = TileProduct16<T, 64, 64, 2, 2, 3, 2, true>;  // (of paired tiles alone)
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
//   64 x 32     up to 256 of these: 146 rows, 768 -> 2304 (216 tiles) 6.4 (128 x 64: 7.7), 96 rows, 4096 -> 4096 (256) 18.4
//               (23.8); 200 rows, 768 -> 2304 (288) 10.9 (7.7), 48 rows, 4096 -> 14336 (448) 40 (36)
//   128 x 64    otherwise, until
//   256 x 128   there are 144 of these: 1,500 rows, 768 -> 2304 (108) 19.1 (15.4), 2,048 rows (144) 19.9 (22.8), 1,024 rows,
//               4096 -> 4096 (128) 72 (61), 1,500 rows (192) 80 (91)
// (Past a whole round of these there is no rule for the last one, as rows() has.)
template <class T, class A, bool GRAD>
hipError_t gated(const GatedArgs& a, hipStream_t s) {
  auto tiles = [&](int t, int m) { return (a.n + t - 1) / t * ((a.f + m - 1) / m); };
  if (a.n <= 32) return gated_few_as<T, A, GRAD>(a, s);
  if (tiles(64, 32) <= 256) return gated_as<T, A, Small<T>, GRAD, kSmallGroups>(a, s);
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

template <class T, class P>
hipError_t rows_as(const ProductArgs& a, hipStream_t s) {
  const int64_t grid = (a.n - a.row0 + P::kRows - 1) / P::kRows * ((a.m + P::kCols - 1) / P::kCols) * a.splits;
  const auto kernel = rows_kernel<T, P>;
  const hipError_t e = allow_lds((const void*)kernel, P::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(P::kThreads), P::kLds, s, a);
  return hipGetLastError();
}

// How a product's tiles are made: the least estimated time, of 256 workgroups at a time, a stage of 64 values of k taking
// a tile 1.26 us (256 x 256) or 0.55 (128 x 128), and the splits' sums 8 bytes a value, written and read at 3.5 TB/s, and a
// launch.  The stages' times were taken with both operands by rows; as they are now a stage of dx takes 1.05 to 1.17 us
// (up to 128 tiles of 256 x 256, 4096 -> 14336) and 1.45 (256 of them), and 0.39 (64 tiles of 128 x 128) to 0.57 (256 and
// more).  (dx's product, us, as the rule has it, in tiles of 128 and in tiles of 256, each without splits: 256 rows,
// 4096 -> 14336 72, 176 and 471, 764 rows 153, 223 and 484, 2,048 rows 352, 484 and 523, 4,096 rows 656, 1,017 and 648,
// 764 rows, 768 -> 2304 20, 35 and 84.)
struct RowsPlan {
  bool wide;  // 256 x 256, or 128 x 128
  int splits;
};
RowsPlan rows_plan(int64_t n, int m, int k) {
  constexpr double kStage[2] = {0.55, 1.26};
  const int64_t stages = k > 0 ? ((int64_t)k + 63) / 64 : 1;
  RowsPlan best = {true, 1};
  double least = 0.0;
  for (int wide = 1; wide >= 0; --wide) {
    const int size = wide ? 256 : 128;
    const int64_t tiles = (n + size - 1) / size * ((m + size - 1) / size);
    if (!wide && !launch_fits(tiles, Middle<HalfBf16, false>::kThreads)) continue;  // (gated_fits has asked for the others)
    const int most = tiles >= 256 ? 1 : 16;
    for (int s = 1; s <= most && (s == 1 || (tiles * s <= 256 && stages / s >= 4)); ++s) {
      const double rounds = (double)((tiles * s + 255) / 256), part = (double)((stages + s - 1) / s);
      const double us = rounds * part * kStage[wide] + (s > 1 ? 8.0 + (double)s * (double)n * m * 8.0 / 3.5e6 : 0.0);
      if (wide && s == 1) least = us;
      if (us < least) {
        least = us;
        best = {wide != 0, s};
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
  if (!plan.wide) {
    e = rows_as<T, Middle<T, false>>(a, s);
  } else {
    // A last round of up to 112 tiles (of 256, one a CU) is left to the next size, where these are at most 448: two rounds.
    // (They may be more, because the rows are cut at whole tile rows: 2,048 rows, 11000 -> 4096, x's gradients 643 us in
    // one launch, 679 with 516 of them.)
    const int64_t n_m = (a.m + 255) / 256, tiles = (a.n + 255) / 256 * n_m, rest = tiles % 256;
    const int64_t whole = (tiles - rest) / n_m * 256;  // rows of the whole rounds
    const int64_t small = (a.n - whole + 127) / 128 * ((a.m + 127) / 128);
    ProductArgs w = a;
    if (a.splits == 1 && rest > 0 && rest <= 112 && whole > 0 && small <= 448) w.n = whole;
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

}  // namespace

// (Where a limit is near, the tiles are 256 x 128 and 256 x 256 by 512 threads, and max_kernel's of 64 rows; rows_plan
// leaves out smaller ones that do not fit.)
bool gated_fits(int64_t n, int k, int f, bool grads) {
  auto blocks = [](int64_t size, int of) { return (size + of - 1) / of; };
  if (!launch_fits(blocks(n, 256) * blocks(f, 128), 512)) return false;
  if (!grads) return true;
  return launch_fits(blocks(gated_cols_at(n) + f, 256), 256) && launch_fits(blocks(n, 64) * blocks(f, 512), 256) &&
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

hipError_t launch_gated_max(const uint16_t* dh, int64_t n, int f, uint32_t* words, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const int64_t all = gated_cols_at(n) + f;
  hipLaunchKernelGGL(clear_kernel, dim3((unsigned)((all + 255) / 256)), dim3(256), 0, stream, words, all);
  uint32_t *const rows = words, *const cols = words + gated_cols_at(n);
  // fewer atomics where there are workgroups enough
  const int64_t n_c = (f + 511) / 512;
  if ((n + 63) / 64 * n_c >= 1024)
    hipLaunchKernelGGL(max_kernel<16>, dim3((unsigned)((n + 63) / 64 * n_c)), dim3(256), 0, stream, dh, n, f, rows, cols);
  else
    hipLaunchKernelGGL(max_kernel<4>, dim3((unsigned)((n + 15) / 16 * n_c)), dim3(256), 0, stream, dh, n, f, rows, cols);
  return hipGetLastError();
}

}  // namespace hpr
