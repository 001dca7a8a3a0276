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
// 16 bytes that are not read again soon: past the caches, which keep what is.
__device__ __forceinline__ void store16_stream(void* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
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
      const float q = LAYER ? (in[c] ? v[c][i] - mean : 0.f) : v[c][i];
      s[0] += q * q;
    }
  sums(s);
  rs = __builtin_amdgcn_rsqf(s[0] * inv_d + eps);
}

// A row per W waves, read once: x and b in, r and y out.  Bound by memory: 53,248 rows of 4096 (1.74 GB) 296 us, 5.9 TB/s
// (304 with stores that stay in the caches; with 13,057 rows, whose inputs still lie in the last cache, 60 and 82).  Small
// calls wait for two dependent sums: 64 rows 4.5 us.
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
      if (a.r) store16_stream(a.r + row * a.d + col[c], narrow<T>(r[c]));
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
      store16_stream(a.y + row * a.d + col[c], narrow<T>(y));
    }
  }
}

// Rows in turn by a fixed number of workgroups, each of which keeps its rows' sums over columns in registers:
//   sums 0 and 1: dy s, and t times dx or, where the gate is the row's own, times scale gate dx;  2 and 3: the same
//   without s and t.
// The next row is on its way while one is worked on, and the vectors stay in registers, up to 8,192 values (C = 1).
//
// Bound by memory, with vector instructions for two fifths of the time, where that fits the registers: 53,248 rows of
// 4096 (2.6 GB) 525 to 540 us, 4.9 TB/s (a copy reaches 5.1), from checkpoints 475.  More waves a row, not more chunks a
// lane: two rows' tensors and the sums fill the registers of C = 1.  128 registers, four waves a SIMD, hold RMS norm up to
// 8,192 values (from checkpoints above 4,096 all but 2 to 4), with gates of rows up to 2,048 (129 of one form).
// Layer norm has twice the sums and takes 122 to 159 up to 2,048 values: past 128 (with gates of rows; in bf16 above 512
// values; above 1,024) three workgroups are on a CU, and the launch's 1,024 are a round and a third.  Above 2,048 values,
// where a workgroup's size leaves 128, layer norm spills 23 to 67 of a lane's registers, RMS with gates of rows up to 28,
// and above 8,192 values every form 41 to 150.  53.5 million values in bf16, us, RMS and layer norm: rows of 512 131 and
// 140, 768 137 and 167 (fp16 138 and 150), 1024 134 and 154, 2048 135 and 161, 4096 135 and 245, 8192 139 and 473, 16384
// 353 and 827; with gates of rows 768 179 and 201, 2048 177 and 195, 4096 178 and 426, 8192 257 and 635.
//
// Rows are read and written through buffers of their own length, 0 for what there is not: values past the row, rows
// past the last and tensors that are not there read as zeros and are not written, without a branch (with masks and
// branches a third of the instructions were moves).  Zeros go through the formulas as zeros: of LAYER's mean alone
// the lanes past the row are kept out.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_of(const void* base, int64_t first, int64_t bytes, bool there) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base)) + first, (short)0,
                                           there && base ? (int)bytes : 0, 0x00020000);
}
__device__ __forceinline__ u32x4 read16(__amdgpu_buffer_rsrc_t r, int at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
}
__device__ __forceinline__ void write16(__amdgpu_buffer_rsrc_t r, int at, u32x4 v) {
  typedef unsigned int v4u __attribute__((ext_vector_type(4)));
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), r, at, 0, 2);  // nt, as store16_stream
}

template <int C>
struct RowLoads {
  u32x4 dr[C], dy[C], gate[C];
  u32x4 x[C], b[C];       // of packed rows the codes alone
  uint32_t ex[C], eb[C];  // and their exponents
};

template <class T, bool LAYER, bool PACKED, bool GATE_ROWS, int W, int C>
__device__ __forceinline__ void norm_bwd_rows(const NormArgs& a) {
  typedef Layout<W, C> L;
  constexpr int kSums = LAYER ? 4 : 2;
  constexpr bool kHold = C == 1;
  __shared__ float lds[2][L::kWaves][4];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowSums<W, L::kWaves> sums = {lds, wave, 0};
  const float inv_d = 1.f / (float)a.d;
  const int blocks = (a.d + 31) / 32;
  const bool has_b = PACKED ? a.b_codes != nullptr : a.b != nullptr;
  int col[C];
  bool live[C];
  float total[kSums][C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = 8 * ((wave % W) * 64 + lane + 64 * W * c);
    live[c] = col[c] < a.d;
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) total[k][c][i] = 0.f;
  }
  // w;  scale pw, and scale pc, times the gate where it is shared
  auto vectors = [&](int c, float (&w)[8], float (&pw)[8], float (&pc)[8]) __attribute__((always_inline)) {
    float g[8];
    vector8<T>(live[c] ? a.w : nullptr, col[c], 0.f, w);
    vector8<T>(live[c] ? a.pw : nullptr, col[c], 1.f, pw);
    vector8<T>(LAYER && live[c] ? a.pc : nullptr, col[c], 0.f, pc);
    vector8<T>(!GATE_ROWS && live[c] ? a.gate : nullptr, col[c], 1.f, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float by = a.scale * g[i];
      pw[i] *= by;
      pc[i] *= by;
    }
  };
  float w_[kHold ? C : 1][8], pw_[kHold ? C : 1][8], pc_[kHold ? C : 1][8];
  if constexpr (kHold) {
#pragma unroll
    for (int c = 0; c < C; ++c) vectors(c, w_[c], pw_[c], pc_[c]);
  }
  const int64_t bytes = 2 * (int64_t)a.d;
  auto load = [&](int64_t row, RowLoads<C>& l) __attribute__((always_inline)) {
    const bool there = row < a.n;
    const auto dr = row_of(a.dr, row * bytes, bytes, there), dy = row_of(a.dy, row * bytes, bytes, there);
    const auto gate = row_of(GATE_ROWS ? a.gate : nullptr, row * bytes, bytes, there);
    const void *xp = a.x, *bp = a.b;
    if constexpr (PACKED) xp = a.x_codes, bp = a.b_codes;
    const auto x = row_of(xp, PACKED ? row * a.d : 2 * row * a.x_ld, PACKED ? a.d : bytes, there);
    const auto b = row_of(bp, PACKED ? row * a.d : 2 * row * a.b_ld, PACKED ? a.d : bytes, there);
    const auto ex = row_of(PACKED ? a.x_exps : nullptr, row * blocks, blocks, there);
    const auto eb = row_of(PACKED ? a.b_exps : nullptr, row * blocks, blocks, there);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      l.dr[c] = read16(dr, 2 * col[c]);
      l.dy[c] = read16(dy, 2 * col[c]);
      if constexpr (GATE_ROWS) l.gate[c] = read16(gate, 2 * col[c]);
      if constexpr (PACKED) {
        const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(x, col[c], 0, 0));
        const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(b, col[c], 0, 0));
        l.x[c][0] = v.x, l.x[c][1] = v.y;
        l.b[c][0] = u.x, l.b[c][1] = u.y;
        l.ex[c] = __builtin_amdgcn_raw_buffer_load_b8(ex, col[c] / 32, 0, 0);
        l.eb[c] = __builtin_amdgcn_raw_buffer_load_b8(eb, col[c] / 32, 0, 0);
      } else {
        l.x[c] = read16(x, 2 * col[c]);
        l.b[c] = read16(b, 2 * col[c]);
      }
    }
  };
  auto rows_of = [&](const u32x4& v, uint32_t e, float (&f)[8]) __attribute__((always_inline)) {
    if constexpr (PACKED) code_values(uint2{v[0], v[1]}, e, f);
    else widen<T>(v, f);
  };
  RowLoads<C> next;
  const int64_t first = (int64_t)blockIdx.x * L::kRows, stride = (int64_t)gridDim.x * L::kRows;
  if constexpr (kHold) load(first + wave / W, next);
  // (the same number of turns for every wave of the workgroup: the sums have barriers)
  for (int64_t row0 = first; row0 < a.n; row0 += stride) {
    const int64_t row = row0 + wave / W;
    const bool there = row < a.n;
    if constexpr (!kHold) load(row, next);
    float r[C][8], t[C][8], e[C][8], dr[C][8], g[GATE_ROWS ? C : 1][8];  // t: b, then its normalised values; e: dy
#pragma unroll
    for (int c = 0; c < C; ++c) {
      rows_of(next.x[c], next.ex[c], r[c]);
      rows_of(next.b[c], next.eb[c], t[c]);
      widen<T>(next.dr[c], dr[c]);
      widen<T>(next.dy[c], e[c]);
      if constexpr (GATE_ROWS) widen<T>(next.gate[c], g[c]);
    }
    if constexpr (kHold) load(row + stride, next);
    auto at_c = [&](int c, float (&w)[8], float (&pw)[8], float (&pc)[8]) __attribute__((always_inline)) {
      if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = w_[c][i], pw[i] = pw_[c][i], pc[i] = pc_[c][i];
      } else {
        vectors(c, w, pw, pc);
      }
    };
    float mean_b = 0.f, rs_b = 1.f;
    if (a.pw) statistics<LAYER, C>(t, live, inv_d, a.eps, sums, mean_b, rs_b);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[8], pw[8], pc[8];
      at_c(c, w, pw, pc);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        t[c][i] = LAYER ? (live[c] ? (t[c][i] - mean_b) * rs_b : 0.f) : t[c][i] * rs_b;
        const float p = LAYER ? t[c][i] * pw[i] + pc[i] : t[c][i] * pw[i];
        r[c][i] += GATE_ROWS ? g[c][i] * p : p;
      }
    }
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
    float s[LAYER ? 3 : 2];  // of (r - mean)^2, e (r - mean), e
#pragma unroll
    for (float& v : s) v = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[8], pw[8], pc[8];
      at_c(c, w, pw, pc);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = LAYER ? (live[c] ? r[c][i] - mean : 0.f) : r[c][i], v = e[c][i] * w[i];
        r[c][i] = q;
        s[0] += q * q;
        s[1] += v * q;
        if constexpr (LAYER) s[2] += v;
      }
    }
    sums(s);
    const float rs = __builtin_amdgcn_rsqf(s[0] * inv_d + a.eps);
    const float along = s[1] * inv_d * rs;
    float base = 0.f;
    if constexpr (LAYER) base = s[2] * inv_d;
    const auto dx = row_of(a.dx, row * bytes, bytes, there), db = row_of(a.db, row * bytes, bytes, there);
    const auto dgate = row_of(GATE_ROWS ? a.dgate_rows : nullptr, row * bytes, bytes, there);
    float back[2] = {0.f, 0.f};  // sums of f t, f
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[8], pw[8], pc[8], dg[8];
      at_c(c, w, pw, pc);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = r[c][i] * rs;
        total[0][c][i] += e[c][i] * q;
        if constexpr (LAYER) total[2][c][i] += e[c][i];
        const float d = dr[c][i] + (LAYER ? e[c][i] * w[i] - base - q * along : e[c][i] * w[i] - q * along) * rs;
        dr[c][i] = d;  // dx from here on
        float f = d * pw[i], of = d;
        if constexpr (GATE_ROWS) {
          f *= g[c][i];
          of *= a.scale * g[c][i];
          dg[i] = d * (LAYER ? t[c][i] * pw[i] + pc[i] : t[c][i] * pw[i]);
        }
        total[1][c][i] += of * t[c][i];
        if constexpr (LAYER) total[3][c][i] += of;
        back[0] += f * t[c][i];
        if constexpr (LAYER) back[1] += live[c] ? f : 0.f;
        r[c][i] = f;
      }
      write16(dx, 2 * col[c], narrow<T>(dr[c]));
      if constexpr (GATE_ROWS) write16(dgate, 2 * col[c], narrow<T>(dg));
    }
    if (!has_b) continue;
    if (a.pw) sums(back);
    const float along_b = a.pw ? back[0] * inv_d : 0.f, base_b = LAYER && a.pw ? back[1] * inv_d : 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = LAYER ? (r[c][i] - base_b - t[c][i] * along_b) * rs_b : (r[c][i] - t[c][i] * along_b) * rs_b;
      write16(db, 2 * col[c], narrow<T>(v));
    }
  }
  // the workgroup's rows join in LDS, one wave row after another
  float* part = a.part + (int64_t)blockIdx.x * kSums * a.d;
  if constexpr (L::kRows > 1) {
    __shared__ float joined[kSums][512 * W * C];
    for (int q = 0; q < L::kRows; ++q) {
      if (wave / W == q) {
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
          for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
              f32x4* to = reinterpret_cast<f32x4*>(&joined[k][col[c] + i]);
              f32x4 v = {total[k][c][i], total[k][c][i + 1], total[k][c][i + 2], total[k][c][i + 3]};
              *to = q == 0 ? v : *to + v;
            }
      }
      __syncthreads();
    }
    for (int i = 4 * threadIdx.x; i < kSums * 512 * W * C; i += 4 * L::kThreads) {
      const int k = i / (512 * W * C), c = i % (512 * W * C);
      if (c < a.d)
        *reinterpret_cast<f32x4*>(part + (int64_t)k * a.d + c) = *reinterpret_cast<const f32x4*>(&joined[k][c]);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!live[c]) continue;
      float* to = part + (int64_t)k * a.d + col[c];
      *reinterpret_cast<f32x4*>(to) = f32x4{total[k][c][0], total[k][c][1], total[k][c][2], total[k][c][3]};
      *reinterpret_cast<f32x4*>(to + 4) = f32x4{total[k][c][4], total[k][c][5], total[k][c][6], total[k][c][7]};
    }
}

// (Eight waves a row are two workgroups a CU with 128 registers, which some forms spill for: see above.)
template <class T, bool LAYER, bool PACKED, bool GATE_ROWS, int W, int C>
__global__ __launch_bounds__((Layout<W, C>::kThreads), W == 8 ? 4 : 1) void norm_bwd_kernel(NormArgs a) {
  norm_bwd_rows<T, LAYER, PACKED, GATE_ROWS, W, C>(a);
}

// The workgroups' sums of 16 columns, in their order within 256 runs of workgroups, then over the runs; and the
// gradients that come of them.  Reads 8 or 16 bytes a column and workgroup of the gradients' kernel: 4096 columns of 512
// workgroups (17 MB) 8.9 us, 768 columns of 1,024 (13 MB) 10.7 (in 64 runs: 9.0 and 13.1), most of it start and latency.
constexpr int kJoinRuns = 256;
template <class T, bool LAYER>
__global__ __launch_bounds__(4 * kJoinRuns) void norm_join_kernel(NormArgs a) {
  constexpr int kSums = LAYER ? 4 : 2, kParts = 4 * kJoinRuns / (16 * kSums), kOf = kJoinRuns / kParts;
  __shared__ float lds[kJoinRuns][kSums][16];
  const int q = threadIdx.x & 3, run = threadIdx.x >> 2;
  const int c = (int)blockIdx.x * 16 + 4 * q;
  f32x4 v[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (c < a.d) {
#pragma unroll 4
    for (int64_t g = a.parts * run / kJoinRuns; g < a.parts * (run + 1) / kJoinRuns; ++g)
#pragma unroll
      for (int k = 0; k < kSums; ++k)
        v[k] += *reinterpret_cast<const f32x4*>(a.part + (g * kSums + k) * a.d + c);
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) *reinterpret_cast<f32x4*>(&lds[run][k][4 * q]) = v[k];
  __syncthreads();
  const int j = threadIdx.x & 15, of = (threadIdx.x >> 4) % kSums, part = threadIdx.x / (16 * kSums);
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < kOf; ++w) sum += lds[part * kOf + w][of][j];
  __syncthreads();
  lds[part][of][j] = sum;
  __syncthreads();
  const int to = (int)blockIdx.x * 16 + j;
  if (threadIdx.x >= 16 || to >= a.d) return;
  float s[kSums];
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    s[k] = 0.f;
#pragma unroll
    for (int w = 0; w < kParts; ++w) s[k] += lds[w][k][j];
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

template <int N>
using Int = std::integral_constant<int, N>;

// W and C of a row of d values in the forward, and in the gradients, which hold more of a column in registers.
template <class F>
hipError_t by_dim(int d, F&& f) {
  if (d <= 512) return f(Int<1>(), Int<1>());
  if (d <= 1024) return f(Int<1>(), Int<2>());
  if (d <= 2048) return f(Int<2>(), Int<2>());
  if (d <= 4096) return f(Int<4>(), Int<2>());
  if (d <= 8192) return f(Int<8>(), Int<2>());
  return f(Int<8>(), Int<4>());
}
template <class F>
hipError_t by_dim_bwd(int d, F&& f) {
  if (d <= 512) return f(Int<1>(), Int<1>());
  if (d <= 1024) return f(Int<2>(), Int<1>());
  if (d <= 2048) return f(Int<4>(), Int<1>());
  if (d <= 4096) return f(Int<8>(), Int<1>());
  if (d <= 8192) return f(Int<16>(), Int<1>());
  return f(Int<16>(), Int<2>());
}
int rows_of_group(int d) { return d <= 512 ? 4 : d <= 1024 ? 2 : 1; }  // Layout::kRows of the gradients

// Workgroups of the gradients: four a CU, or two, where their registers are as many as RMS norm's.  (Above 4,096 values,
// 16 waves, one is on a CU, and these are two rounds.)
int groups_most(int d) { return d <= 2048 ? 1024 : 512; }

template <class T, bool LAYER>
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) {
  return by_dim(a.d, [&](auto w, auto c) {
    typedef Layout<w(), c()> L;
    hipLaunchKernelGGL((norm_fwd_kernel<T, LAYER, w(), c()>), dim3((unsigned)((a.n + L::kRows - 1) / L::kRows)),
                       dim3(L::kThreads), 0, s, a);
    return hipGetLastError();
  });
}

template <class T, bool LAYER, bool PACKED, bool GATE_ROWS>
hipError_t norm_bwd(const NormArgs& a, hipStream_t s) {
  const hipError_t e = by_dim_bwd(a.d, [&](auto w, auto c) {
    typedef Layout<w(), c()> L;
    if (a.parts == 0) return hipSuccess;
    hipLaunchKernelGGL((norm_bwd_kernel<T, LAYER, PACKED, GATE_ROWS, w(), c()>), dim3((unsigned)a.parts),
                       dim3(L::kThreads), 0, s, a);
    return hipGetLastError();
  });
  if (e != hipSuccess || !(a.dw || a.dc || a.dpw || a.dpc || a.dgate)) return e;
  hipLaunchKernelGGL((norm_join_kernel<T, LAYER>), dim3((unsigned)((a.d + 15) / 16)), dim3(4 * kJoinRuns), 0, s, a);
  return hipGetLastError();
}

template <class T, bool LAYER>
hipError_t norm_bwd_of(const NormArgs& a, hipStream_t s) {
  if (a.x_codes) return a.gate_rows ? norm_bwd<T, LAYER, true, true>(a, s) : norm_bwd<T, LAYER, true, false>(a, s);
  return a.gate_rows ? norm_bwd<T, LAYER, false, true>(a, s) : norm_bwd<T, LAYER, false, false>(a, s);
}

}  // namespace

// Workgroups of the gradients, whose sums are kept apart.
int64_t norm_parts(int64_t n, int d) {
  const int64_t per = rows_of_group(d), groups = (n + per - 1) / per;
  return groups < groups_most(d) ? groups : groups_most(d);
}

bool norm_fits(int64_t n, int d) {
  const int64_t per = d <= 1024 ? 4 : d <= 2048 ? 2 : 1;  // Layout::kRows of the forward, which has more workgroups
  return launch_fits((n + per - 1) / per, d <= 4096 ? 256 : 512);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  if (a.f16) return a.layer ? norm_fwd<HalfF16, true>(a, stream) : norm_fwd<HalfF16, false>(a, stream);
  return a.layer ? norm_fwd<HalfBf16, true>(a, stream) : norm_fwd<HalfBf16, false>(a, stream);
}

hipError_t launch_norm_bwd(NormArgs a, hipStream_t stream) {
  a.parts = norm_parts(a.n, a.d);
  if (a.f16) return a.layer ? norm_bwd_of<HalfF16, true>(a, stream) : norm_bwd_of<HalfF16, false>(a, stream);
  return a.layer ? norm_bwd_of<HalfBf16, true>(a, stream) : norm_bwd_of<HalfBf16, false>(a, stream);
}

}  // namespace hpr
