// Rotation of queries and keys by their position.
//
// With c and s the position's row of the cosine and sine tables, values j and j + rot / 2 of every
// head turn together:  (x_j c_j - x_{j + rot/2} s_j,  x_{j + rot/2} c_j + x_j s_j);  values past
// rot pass through.  The gradient is the rotation back (s negated).  A position outside the table
// gives NaN.
//
// Bound by memory.  A thread takes 8 values of both halves of one head (two 16-byte loads and
// stores); queries and keys go in one launch.
#include "common.h"
#include "half.h"
#include "kernels.h"

namespace hpr {

namespace {

constexpr int kRotThreads = 256;

template <class T>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, int pairs, int items) {
  const int64_t w = (int64_t)blockIdx.x * kRotThreads + threadIdx.x;
  const int64_t t = w / items;
  if (t >= a.n) return;
  int i = (int)(w - t * items);
  // items of a row: per head, `pairs` rotated chunk pairs, then the chunks that pass through
  const int per_head = pairs + (a.dim - a.rot) / 8;
  int h = i / per_head;
  i -= h * per_head;
  const int which = h >= a.heads[0];
  if (which) h -= a.heads[0];
  const uint16_t* src = a.x[which] + t * a.row[which] + h * a.head[which];
  uint16_t* dst = a.out[which] + (t * a.heads[which] + h) * a.dim;
  if (i >= pairs) {
    const int d = a.rot + 8 * (i - pairs);
    *reinterpret_cast<u32x4*>(dst + d) = load16(src + d);
    return;
  }
  const int half = a.rot / 2, d = 8 * i;
  const int32_t p = a.pos[t];
  const bool in = p >= 0 && p < a.n_pos;
  const float* cp = a.cosp + (in ? p : 0) * (int64_t)half + d;
  const float* sp = a.sinp + (in ? p : 0) * (int64_t)half + d;
  const u32x4 u = load16(src + d), v = load16(src + half + d);
  u32x4 ou, ov;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 c = *reinterpret_cast<const float2*>(cp + 2 * e);
    float2 s = *reinterpret_cast<const float2*>(sp + 2 * e);
    if (a.inverse) s.x = -s.x, s.y = -s.y;
    const float u0 = T::lo(u[e]), u1 = T::hi(u[e]), v0 = T::lo(v[e]), v1 = T::hi(v[e]);
    const float bad = __builtin_nanf("");
    ou[e] = T::pack(in ? u0 * c.x - v0 * s.x : bad, in ? u1 * c.y - v1 * s.y : bad);
    ov[e] = T::pack(in ? v0 * c.x + u0 * s.x : bad, in ? v1 * c.y + u1 * s.y : bad);
  }
  *reinterpret_cast<u32x4*>(dst + d) = ou;
  *reinterpret_cast<u32x4*>(dst + half + d) = ov;
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  const int pairs = a.rot / 16;
  const int items = (a.heads[0] + a.heads[1]) * (pairs + (a.dim - a.rot) / 8);
  const int64_t grid = (a.n * items + kRotThreads - 1) / kRotThreads;
  if (grid == 0) return hipSuccess;
  if (a.f16)
    hipLaunchKernelGGL(rotary_kernel<HalfF16>, dim3((unsigned)grid), dim3(kRotThreads), 0, stream, a,
                       pairs, items);
  else
    hipLaunchKernelGGL(rotary_kernel<HalfBf16>, dim3((unsigned)grid), dim3(kRotThreads), 0, stream,
                       a, pairs, items);
  return hipGetLastError();
}

}  // namespace hpr
