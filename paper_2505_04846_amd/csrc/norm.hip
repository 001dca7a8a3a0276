// The norms around a block of an encoder, with its gate, residual scale and residual sum, and their gradients.
//
// For a row x of the residual stream and a row b of the block's output:
//   p = N(b; pw, pc)      (b itself without a norm after the block)
//   r = x + scale * gate * p      (x itself without a block)
//   y = N(r; w, c)
// where N(v; w, c) is (v - mean) / sqrt(variance + eps) * w + c, or v / sqrt(mean square + eps) * w.
//
// Gradients, for dr and dy: with the normalised rows s = (r - mean) / sigma and t (of b), e = dy w,
//   dx = dr + (e - mean(e) - s mean(e s)) / sigma      (without mean(e) where the norm takes no mean)
//   dp = scale gate dx,   f = dp pw,   db = (f - mean(f) - t mean(f t)) / sigma_b
//   dw = sum dy s,  dc = sum dy,  dpw = sum dp t,  dpc = sum dp,  dgate = scale dx p (summed where it is shared).
// They need x and b alone: the statistics are formed again, r is not kept, and both are the exact ones, whether the
// rows come in 16 bits or from a checkpoint in 8.
//
// Everything is in 32 bits, from the rows as read to the outputs, each rounded once (y from the unrounded r).  A
// row lies in the registers of its W waves; means are taken off before squares are summed (a second pass over
// registers, not over memory).
#include <type_traits>

#include "checkpoint.h"
#include "common.h"
#include "half.h"
#include "kernels.h"

namespace hpr {

namespace {

// ---- sums over a row ----------------------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
// Sum over the wave, in every lane: 16 lanes by moves between them, then the four sixteens.
__device__ __forceinline__ float sum_of_wave(float v) {
  v += dpp<0xb1>(v);   // lane ^ 1
  v += dpp<0x4e>(v);   // lane ^ 2
  v += dpp<0x141>(v);  // 7 - lane, of eight
  v += dpp<0x140>(v);  // 15 - lane
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// Sums over a row of W waves, in every lane.  `turn` changes with every call, so that one barrier is enough.
template <int W, int WAVES>
struct RowSums {
  float (*lds)[WAVES][4];  // [2]
  int wave, turn;
  template <int K>
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    static_assert(K <= 4, "");
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = sum_of_wave(v[k]);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) lds[turn][wave][k] = v[k];
      }
      __syncthreads();
      const int first = wave / W * W;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        v[k] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v[k] += lds[turn][first + w][k];
      }
      turn ^= 1;
    }
  }
};

template <class T>
__device__ __forceinline__ void widen(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = T::lo(v[i]);
    f[2 * i + 1] = T::hi(v[i]);
  }
}
template <class T>
__device__ __forceinline__ u32x4 narrow(const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = T::pack(f[2 * i], f[2 * i + 1]);
  return v;
}
// Eight values of a vector of d at col, `other` without one.
template <class T>
__device__ __forceinline__ void vector8(const uint16_t* p, int64_t at, float other, float (&f)[8]) {
  if (p) {
    widen<T>(load16(p + at), f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = other;
  }
}

// How the rows lie in a workgroup: W waves a row, C chunks of 8 values a lane.
template <int W, int C>
struct Layout {
  static constexpr int kWaves = W > 4 ? W : 4, kThreads = 64 * kWaves, kRows = kWaves / W;
};

// Mean (0 without LAYER) and 1 / sigma of the rows v; lanes past the row hold nothing.
template <bool LAYER, int C, class Sums>
__device__ __forceinline__ void statistics(const float (&v)[C][8], const bool (&in)[C], float inv_d, float eps,
                                           Sums& sums, float& mean, float& rs) {
  float s[1] = {0.f};
  mean = 0.f;
  if constexpr (LAYER) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[c][i];
    sums(s);
    mean = s[0] * inv_d;
    s[0] = 0.f;
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = in[c] ? v[c][i] - mean : 0.f;
      s[0] += q * q;
    }
  sums(s);
  rs = 1.f / __builtin_sqrtf(s[0] * inv_d + eps);
}

template <class T, bool LAYER, int W, int C>
__global__ __launch_bounds__((Layout<W, C>::kThreads)) void norm_fwd_kernel(NormArgs a) {
  typedef Layout<W, C> L;
  __shared__ float lds[2][L::kWaves][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  RowSums<W, L::kWaves> sums = {lds, wave, 0};
  const int64_t row = (int64_t)blockIdx.x * L::kRows + wave / W;
  const float inv_d = 1.f / (float)a.d;
  int col[C];
  bool in[C];
  float r[C][8], b[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = 8 * ((wave % W) * 64 + lane + 64 * W * c);
    in[c] = col[c] < a.d && row < a.n;
    u32x4 x = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
    if (in[c]) {
      x = load16(a.x + row * a.x_ld + col[c]);
      if (a.b) v = load16(a.b + row * a.b_ld + col[c]);
    }
    widen<T>(x, r[c]);
    widen<T>(v, b[c]);
  }
  if (a.b) {
    float mean = 0.f, rs = 1.f;
    if (a.pw) statistics<LAYER, C>(b, in, inv_d, a.eps, sums, mean, rs);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      float w[8], o[8], g[8];
      vector8<T>(a.pw, col[c], 1.f, w);
      vector8<T>(LAYER ? a.pc : nullptr, col[c], 0.f, o);
      vector8<T>(a.gate, (a.gate_rows ? row * a.d : 0) + col[c], 1.f, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) r[c][i] += a.scale * g[i] * ((b[c][i] - mean) * rs * w[i] + o[i]);
      if (a.r) *reinterpret_cast<u32x4*>(a.r + row * a.d + col[c]) = narrow<T>(r[c]);
    }
  }
  if (a.y) {
    float mean, rs;
    statistics<LAYER, C>(r, in, inv_d, a.eps, sums, mean, rs);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      float w[8], o[8], y[8];
      vector8<T>(a.w, col[c], 1.f, w);
      vector8<T>(LAYER ? a.c : nullptr, col[c], 0.f, o);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = (r[c][i] - mean) * rs * w[i] + o[i];
      *reinterpret_cast<u32x4*>(a.y + row * a.d + col[c]) = narrow<T>(y);
    }
  }
}

// Rows in turn by a fixed number of workgroups, each of which keeps its rows' sums over columns in registers:
//   sums 0 and 1: dy s and (of dx, or of dp where the gate is the row's own) times t;  2 and 3: the same without s, t.
template <class T, bool LAYER, bool PACKED, int W, int C>
__global__ __launch_bounds__((Layout<W, C>::kThreads)) void norm_bwd_kernel(NormArgs a) {
  typedef Layout<W, C> L;
  constexpr int kSums = LAYER ? 4 : 2;
  __shared__ float lds[2][L::kWaves][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  RowSums<W, L::kWaves> sums = {lds, wave, 0};
  const float inv_d = 1.f / (float)a.d;
  const int blocks = (a.d + 31) / 32;
  const bool has_b = PACKED ? a.b_codes != nullptr : a.b != nullptr;
  int col[C];
  float total[kSums][C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = 8 * ((wave % W) * 64 + lane + 64 * W * c);
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) total[k][c][i] = 0.f;
  }
  // (the same number of turns for every wave of the workgroup: the sums have barriers)
  for (int64_t row0 = (int64_t)blockIdx.x * L::kRows; row0 < a.n; row0 += (int64_t)gridDim.x * L::kRows) {
    const int64_t row = row0 + wave / W;
    bool in[C];
    float r[C][8], t[C][8], e[C][8], dr[C][8];  // t: b, then its normalised values; e: dy
#pragma unroll
    for (int c = 0; c < C; ++c) {
      in[c] = col[c] < a.d && row < a.n;
      const int64_t at = row * a.d + col[c];
      u32x4 x = {0u, 0u, 0u, 0u}, b = {0u, 0u, 0u, 0u}, vr = {0u, 0u, 0u, 0u}, vy = {0u, 0u, 0u, 0u};
      if (in[c]) {
        if constexpr (PACKED) {
          const int64_t block = row * blocks + col[c] / 32;
          x = unpack8<T>(*reinterpret_cast<const uint2*>(a.x_codes + at), a.x_exps[block]);
          if (has_b) b = unpack8<T>(*reinterpret_cast<const uint2*>(a.b_codes + at), a.b_exps[block]);
        } else {
          x = load16(a.x + row * a.x_ld + col[c]);
          if (has_b) b = load16(a.b + row * a.b_ld + col[c]);
        }
        if (a.dr) vr = load16(a.dr + at);
        if (a.dy) vy = load16(a.dy + at);
      }
      widen<T>(x, r[c]);
      widen<T>(b, t[c]);
      widen<T>(vr, dr[c]);
      widen<T>(vy, e[c]);
    }
    float mean_b = 0.f, rs_b = 1.f;
    if (has_b) {
      if (a.pw) statistics<LAYER, C>(t, in, inv_d, a.eps, sums, mean_b, rs_b);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (!in[c]) continue;
        float w[8], o[8], g[8];
        vector8<T>(a.pw, col[c], 1.f, w);
        vector8<T>(LAYER ? a.pc : nullptr, col[c], 0.f, o);
        vector8<T>(a.gate, (a.gate_rows ? row * a.d : 0) + col[c], 1.f, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          t[c][i] = (t[c][i] - mean_b) * rs_b;
          r[c][i] += a.scale * g[i] * (t[c][i] * w[i] + o[i]);
        }
      }
    }
    if (a.dy) {
      float mean = 0.f;
      if constexpr (LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) s[0] += r[c][i];
        sums(s);
        mean = s[0] * inv_d;
      }
      float s[3] = {0.f, 0.f, 0.f};  // of (r - mean)^2, e (r - mean), e
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float w[8];
        vector8<T>(in[c] ? a.w : nullptr, col[c], 1.f, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float q = in[c] ? r[c][i] - mean : 0.f, v = e[c][i] * w[i];
          r[c][i] = q;
          s[0] += q * q;
          s[1] += v * q;
          s[2] += v;
        }
      }
      sums(s);
      const float rs = 1.f / __builtin_sqrtf(s[0] * inv_d + a.eps);
      const float along = s[1] * inv_d * rs, base = LAYER ? s[2] * inv_d : 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float w[8];
        vector8<T>(in[c] ? a.w : nullptr, col[c], 1.f, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float q = r[c][i] * rs;
          total[0][c][i] += e[c][i] * q;
          if constexpr (LAYER) total[2][c][i] += e[c][i];
          dr[c][i] += (e[c][i] * w[i] - base - q * along) * rs;
        }
      }
    }
    // dr is dx from here on
    float s[2] = {0.f, 0.f};  // of f t, f
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      const int64_t at = row * a.d + col[c];
      if (a.dx) *reinterpret_cast<u32x4*>(a.dx + at) = narrow<T>(dr[c]);
      if (!has_b) continue;
      float w[8], o[8], g[8], dg[8];
      vector8<T>(a.pw, col[c], 1.f, w);
      vector8<T>(LAYER ? a.pc : nullptr, col[c], 0.f, o);
      vector8<T>(a.gate, (a.gate_rows ? at - col[c] : 0) + col[c], 1.f, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float dp = a.scale * g[i] * dr[c][i], f = dp * w[i];
        dg[i] = a.scale * dr[c][i] * (t[c][i] * w[i] + o[i]);
        const float of = a.gate_rows ? dp : dr[c][i];
        total[1][c][i] += of * t[c][i];
        if constexpr (LAYER) total[3][c][i] += of;
        s[0] += f * t[c][i];
        s[1] += f;
        r[c][i] = f;
      }
      if (a.dgate_rows) *reinterpret_cast<u32x4*>(a.dgate_rows + at) = narrow<T>(dg);
    }
    if (!has_b) continue;
    if (a.pw) sums(s);
    const float along = a.pw ? s[0] * inv_d : 0.f, base = LAYER && a.pw ? s[1] * inv_d : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c] || !a.db) continue;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (r[c][i] - base - t[c][i] * along) * rs_b;
      *reinterpret_cast<u32x4*>(a.db + row * a.d + col[c]) = narrow<T>(v);
    }
  }
  float* part = a.part + ((int64_t)blockIdx.x * L::kRows + wave / W) * kSums * a.d;
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (col[c] >= a.d) continue;
      float* to = part + (int64_t)k * a.d + col[c];
      *reinterpret_cast<f32x4*>(to) = f32x4{total[k][c][0], total[k][c][1], total[k][c][2], total[k][c][3]};
      *reinterpret_cast<f32x4*>(to + 4) = f32x4{total[k][c][4], total[k][c][5], total[k][c][6], total[k][c][7]};
    }
}

// The groups' sums of 64 columns, in their order within 16 runs of groups, then over the runs; and the gradients
// that come of them.
template <class T, bool LAYER>
__global__ __launch_bounds__(256) void norm_join_kernel(NormArgs a) {
  constexpr int kSums = LAYER ? 4 : 2;
  __shared__ f32x4 lds[16][kSums][16];
  const int q = threadIdx.x & 15, run = threadIdx.x >> 4;
  const int c = (int)blockIdx.x * 64 + 4 * q;
  f32x4 v[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (c < a.d)
    for (int64_t g = a.parts * run / 16; g < a.parts * (run + 1) / 16; ++g)
#pragma unroll
      for (int k = 0; k < kSums; ++k)
        v[k] += *reinterpret_cast<const f32x4*>(a.part + (g * kSums + k) * a.d + c);
#pragma unroll
  for (int k = 0; k < kSums; ++k) lds[run][k][q] = v[k];
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int j = threadIdx.x, to = (int)blockIdx.x * 64 + j;
  if (to >= a.d) return;
  float s[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    s[k] = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s[k] += lds[w][k][j >> 2][j & 3];
  }
  const float none = LAYER ? s[kSums - 1] : 0.f;  // sum 3
  auto one = [&](const uint16_t* p, float other) { return p ? T::lo(p[to]) : other; };
  auto put = [&](uint16_t* p, float x) {
    if (p) p[to] = (uint16_t)T::pack(x, 0.f);
  };
  put(a.dw, s[0]);
  if constexpr (LAYER) put(a.dc, s[2]);
  const float by = a.gate_rows ? 1.f : a.scale * one(a.gate, 1.f);
  put(a.dpw, by * s[1]);
  put(a.dpc, by * none);
  put(a.dgate, a.scale * (one(a.pw, 1.f) * s[1] + one(LAYER ? a.pc : nullptr, 0.f) * none));
}

// W and C of a row of d values.
template <class F>
hipError_t by_dim(int d, F&& f) {
  if (d <= 512) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  if (d <= 1024) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
  if (d <= 2048) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
  if (d <= 4096) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
  if (d <= 8192) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
}
int rows_of_group(int d) { return d <= 1024 ? 4 : d <= 2048 ? 2 : 1; }  // Layout::kRows

constexpr int kGroups = 1024;  // workgroups of the gradients

template <class T, bool LAYER>
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) {
  return by_dim(a.d, [&](auto w, auto c) {
    typedef Layout<w(), c()> L;
    hipLaunchKernelGGL((norm_fwd_kernel<T, LAYER, w(), c()>), dim3((unsigned)((a.n + L::kRows - 1) / L::kRows)),
                       dim3(L::kThreads), 0, s, a);
    return hipGetLastError();
  });
}

template <class T, bool LAYER, bool PACKED>
hipError_t norm_bwd(const NormArgs& a, hipStream_t s) {
  const hipError_t e = by_dim(a.d, [&](auto w, auto c) {
    typedef Layout<w(), c()> L;
    if (a.parts == 0) return hipSuccess;
    hipLaunchKernelGGL((norm_bwd_kernel<T, LAYER, PACKED, w(), c()>), dim3((unsigned)(a.parts / L::kRows)),
                       dim3(L::kThreads), 0, s, a);
    return hipGetLastError();
  });
  if (e != hipSuccess || !(a.dw || a.dc || a.dpw || a.dpc || a.dgate)) return e;
  hipLaunchKernelGGL((norm_join_kernel<T, LAYER>), dim3((unsigned)((a.d + 63) / 64)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class T>
hipError_t norm_bwd_of(const NormArgs& a, hipStream_t s) {
  if (a.x_codes) return a.layer ? norm_bwd<T, true, true>(a, s) : norm_bwd<T, false, true>(a, s);
  return a.layer ? norm_bwd<T, true, false>(a, s) : norm_bwd<T, false, false>(a, s);
}

}  // namespace

// Groups of rows whose sums the gradients keep apart.
int64_t norm_parts(int64_t n, int d) {
  const int64_t per = rows_of_group(d), groups = (n + per - 1) / per;
  return (groups < kGroups ? groups : kGroups) * per;
}

bool norm_fits(int64_t n, int d) {
  const int64_t per = rows_of_group(d);
  return launch_fits((n + per - 1) / per, d <= 4096 ? 256 : 512);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  if (a.f16) return a.layer ? norm_fwd<HalfF16, true>(a, stream) : norm_fwd<HalfF16, false>(a, stream);
  return a.layer ? norm_fwd<HalfBf16, true>(a, stream) : norm_fwd<HalfBf16, false>(a, stream);
}

hipError_t launch_norm_bwd(NormArgs a, hipStream_t stream) {
  a.parts = norm_parts(a.n, a.d);
  return a.f16 ? norm_bwd_of<HalfF16>(a, stream) : norm_bwd_of<HalfBf16>(a, stream);
}

}  // namespace hpr
