// Rotation of queries and keys by their position.
//
// With c and s the position's row of the cosine and sine tables, values j and j + rot / 2 of every
// head turn together:  (x_j c_j - x_{j + rot/2} s_j,  x_{j + rot/2} c_j + x_j s_j);  values past
// rot pass through.  The gradient is the rotation back (s negated).  A position outside the table
// gives NaN.
//
// Bound by memory: 53,248 rows of 40 heads of 128, 176 us a launch, 6.2 TB/s.  A thread takes 8 values of both
// halves of one head (two 16-byte loads and stores, whole lines together with its neighbours); queries and
// keys go in one launch.
#include "common.h"
#include "half.h"
#include "kernels.h"

namespace hpr {

namespace {

constexpr int kRotThreads = 256;

// STREAM: loads and stores that do not stay in the caches, for calls that are larger than them (53,248
// rows of 40 heads of 128 and their gradients: 364 us, 395-401 us otherwise).
constexpr int64_t kStreamFrom = int64_t(256) << 20;  // bytes in and out

// Items of a row: per head, `pairs` rotated chunk pairs, then the chunks that pass through.
template <class T, bool STREAM>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, uint32_t pairs,
                                                             uint32_t per_head, uint32_t items) {
  const uint32_t w = blockIdx.x * kRotThreads + threadIdx.x;  // below 2^32: see launch_rotary
  const uint32_t in_launch = w / items;
  const int64_t t = a.first + in_launch;
  if (t >= a.n) return;
  uint32_t i = w - in_launch * items;
  uint32_t h = i / per_head;
  i -= h * per_head;
  const int which = h >= (uint32_t)a.heads[0];
  if (which) h -= a.heads[0];
  const uint16_t* src = (which ? a.x[1] : a.x[0]) + t * (which ? a.row[1] : a.row[0]) +
                        h * (which ? a.head[1] : a.head[0]);
  uint16_t* dst = (which ? a.out[1] : a.out[0]) + (t * (which ? a.heads[1] : a.heads[0]) + h) * a.dim;
  if (i >= pairs) {
    const uint32_t d = a.rot + 8 * (i - pairs);
    *reinterpret_cast<u32x4*>(dst + d) = load16(src + d);
    return;
  }
  const int half = a.rot / 2, d = 8 * i;
  const u32x4 u = STREAM ? load16_stream(src + d) : load16(src + d);
  const u32x4 v = STREAM ? load16_stream(src + half + d) : load16(src + half + d);
  const int32_t p = a.pos[t];
  const bool in = p >= 0 && p < a.n_pos;
  const f32x4* cp = reinterpret_cast<const f32x4*>(a.cosp + (in ? p : 0) * (int64_t)half + d);
  const f32x4* sp = reinterpret_cast<const f32x4*>(a.sinp + (in ? p : 0) * (int64_t)half + d);
  u32x4 ou, ov;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x4 c = cp[q];
    f32x4 s = sp[q];
    if (a.inverse) s = -s;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t uw = u[2 * q + e], vw = v[2 * q + e];
      const float u0 = T::lo(uw), u1 = T::hi(uw), v0 = T::lo(vw), v1 = T::hi(vw);
      const float c0 = c[2 * e], c1 = c[2 * e + 1], s0 = s[2 * e], s1 = s[2 * e + 1];
      const float bad = __builtin_nanf("");
      ou[2 * q + e] = T::pack(in ? u0 * c0 - v0 * s0 : bad, in ? u1 * c1 - v1 * s1 : bad);
      ov[2 * q + e] = T::pack(in ? v0 * c0 + u0 * s0 : bad, in ? v1 * c1 + u1 * s1 : bad);
    }
  }
  if constexpr (STREAM) {
    __builtin_nontemporal_store(ou, reinterpret_cast<u32x4*>(dst + d));
    __builtin_nontemporal_store(ov, reinterpret_cast<u32x4*>(dst + half + d));
  } else {
    *reinterpret_cast<u32x4*>(dst + d) = ou;
    *reinterpret_cast<u32x4*>(dst + half + d) = ov;
  }
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream) {
  const uint32_t pairs = a.rot / 16, per_head = pairs + (a.dim - a.rot) / 8;
  const uint32_t items = (a.heads[0] + a.heads[1]) * per_head;
  // one launch, or, where its threads would reach 2^32, one per run of rows
  const int64_t most = ((int64_t(1) << 32) - 2 * kRotThreads) / items;
  for (a.first = 0; a.first < a.n; a.first += most) {
    const int64_t rows = a.n - a.first < most ? a.n - a.first : most;
    const dim3 grid((unsigned)((rows * items + kRotThreads - 1) / kRotThreads));
    RotaryArgs b = a;
    b.n = a.first + rows;
    const bool big = 4 * a.n * (a.heads[0] + a.heads[1]) * a.dim >= kStreamFrom;
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), 0, stream, b, pairs, per_head, items);
    };
    if (a.f16) {
      if (big) launch(rotary_kernel<HalfF16, true>);
      else launch(rotary_kernel<HalfF16, false>);
    } else {
      if (big) launch(rotary_kernel<HalfBf16, true>);
      else launch(rotary_kernel<HalfBf16, false>);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace hpr
