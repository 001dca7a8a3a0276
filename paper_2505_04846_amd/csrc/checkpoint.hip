// Rows packed into 8 bits (checkpoint.h has the format), and read back.
#include "checkpoint.h"

#include "common.h"
#include "half.h"
#include "kernels.h"

namespace hpr {

namespace {

// A lane takes 8 values, four lanes the 32 of a block; a row's blocks are ceil(d / 32), the last one's missing
// values zero.
constexpr int kThreads = 256;

struct At {
  int64_t row;
  int col, block;  // block of the row
};
__device__ __forceinline__ At chunk_at(int64_t i, uint32_t per_row) {
  // (the row of the workgroup's first chunk by a long division, the chunk's own by a short one)
  const int64_t first = i - threadIdx.x, row0 = first / per_row;
  const uint32_t in = (uint32_t)(first - row0 * per_row) + threadIdx.x, more = in / per_row;
  const uint32_t c = in - more * per_row;
  return {row0 + more, (int)c * 8, (int)(c / 4)};
}

template <class T>
__global__ __launch_bounds__(kThreads) void pack_kernel(const uint16_t* x, int64_t x_ld, int64_t n, int d,
                                                        int8_t* codes, uint8_t* exps) {
  const uint32_t blocks = (uint32_t)(d + 31) / 32u;
  const At p = chunk_at((int64_t)blockIdx.x * kThreads + threadIdx.x, 4 * blocks);
  const bool in = p.row < n && p.col < d;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (in) v = load16(x + p.row * x_ld + p.col);
  float f[8];
  uint32_t most = 0;  // of the magnitudes' bits, whose order is the magnitudes'; NaN above infinity
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = T::lo(v[i]);
    f[2 * i + 1] = T::hi(v[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
    most = most > b ? most : b;
  }
#pragma unroll
  for (int s = 1; s <= 2; s <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)most, s);
    most = most > o ? most : o;
  }
  if (!in) return;
  int e = (int)(most >> 23) - 127 - 6;
  const int least = checkpoint_least<T>();
  e = e > least ? e : least;
  const bool finite = most < 0x7f800000u;
  const float inverse = __uint_as_float(finite ? (uint32_t)(127 - e) << 23 : 0u);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float q = __builtin_rintf(f[i] * inverse);
    q = q > 127.f ? 127.f : (q < -127.f ? -127.f : q);
    const uint32_t code = finite ? (uint32_t)(int)q & 255u : 0u;
    w[i >> 2] |= code << (8 * (i & 3));
  }
  *reinterpret_cast<uint2*>(codes + p.row * d + p.col) = uint2{w[0], w[1]};
  if ((threadIdx.x & 3) == 0) exps[p.row * blocks + p.block] = finite ? (uint8_t)(e + 127) : (uint8_t)255;
}

template <class T>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const int8_t* codes, const uint8_t* exps, int64_t n, int d,
                                                          uint16_t* x) {
  const uint32_t blocks = (uint32_t)(d + 31) / 32u;
  const At p = chunk_at((int64_t)blockIdx.x * kThreads + threadIdx.x, 4 * blocks);
  if (p.row >= n || p.col >= d) return;
  *reinterpret_cast<u32x4*>(x + p.row * d + p.col) =
      unpack8<T>(*reinterpret_cast<const uint2*>(codes + p.row * d + p.col), exps[p.row * blocks + p.block]);
}

unsigned grid_of(int64_t n, int d) { return (unsigned)((n * ((d + 31) / 32 * 4) + kThreads - 1) / kThreads); }

}  // namespace

hipError_t launch_checkpoint_pack(const uint16_t* x, int64_t x_ld, int64_t n, int d, bool f16, int8_t* codes,
                                  uint8_t* exps, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const dim3 grid(grid_of(n, d));
  if (f16)
    hipLaunchKernelGGL(pack_kernel<HalfF16>, grid, dim3(kThreads), 0, stream, x, x_ld, n, d, codes, exps);
  else
    hipLaunchKernelGGL(pack_kernel<HalfBf16>, grid, dim3(kThreads), 0, stream, x, x_ld, n, d, codes, exps);
  return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const int8_t* codes, const uint8_t* exps, int64_t n, int d, bool f16, uint16_t* x,
                                    hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const dim3 grid(grid_of(n, d));
  if (f16)
    hipLaunchKernelGGL(unpack_kernel<HalfF16>, grid, dim3(kThreads), 0, stream, codes, exps, n, d, x);
  else
    hipLaunchKernelGGL(unpack_kernel<HalfBf16>, grid, dim3(kThreads), 0, stream, codes, exps, n, d, x);
  return hipGetLastError();
}

}  // namespace hpr
