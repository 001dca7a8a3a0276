// Rows packed into 8 bits (checkpoint.h has the format), and read back.
#include "checkpoint.h"

#include "common.h"
#include "half.h"
#include "kernels.h"

namespace hpr {

namespace {

// A lane takes 8 values, four lanes the 32 of a block; a row's blocks are ceil(d / 32), the last one's missing
// values zero.  To pack, a wave takes RUNS runs of 64 chunks at a time, so that a lane has RUNS loads on their way and
// the wave's 16 RUNS exponents are one store.
//
// Bound by memory: 53,248 rows of 4096 105 us to pack (6.3 TB/s of 661 MB) and 113 to unpack (5.9).
constexpr int kThreads = 256;

// Chunk i of the rows: row, first column, block of the rows (chunks past the last lie in rows past the last).
struct At {
  int64_t row, block;
  int col;
};
template <int RUNS>
struct Chunks {
  int64_t row0;        // of the workgroup's first chunk, by a long division; the others by short ones
  uint32_t in0, per_row;
  __device__ __forceinline__ Chunks(uint32_t blocks) {
    per_row = 4 * blocks;
    const int64_t first = (int64_t)blockIdx.x * (kThreads * RUNS);
    row0 = first / per_row;
    in0 = (uint32_t)(first - row0 * per_row);
  }
  __device__ __forceinline__ At operator()(uint32_t i) const {
    const uint32_t in = in0 + i, more = in / per_row, c = in - more * per_row;
    const int64_t row = row0 + more;
    return {row, row * (per_row / 4) + c / 4, (int)c * 8};
  }
};

template <class T, int RUNS>
__global__ __launch_bounds__(kThreads) void pack_kernel(const uint16_t* x, int64_t x_ld, int64_t n, int d,
                                                        int8_t* codes, uint8_t* exps) {
  const int lane = threadIdx.x & 63;
  const uint32_t blocks = (uint32_t)(d + 31) / 32u, i0 = (threadIdx.x >> 6) * 64u * RUNS;
  const Chunks<RUNS> chunk(blocks);
  At at[RUNS];
  bool in[RUNS];
  u32x4 v[RUNS];
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    at[k] = chunk(i0 + 64u * k + lane);
    in[k] = at[k].row < n && at[k].col < d;
    v[k] = u32x4{0u, 0u, 0u, 0u};
    if (in[k]) v[k] = load16_stream(x + at[k].row * x_ld + at[k].col);
  }
  uint32_t mine = 0;  // the exponent of the wave's block `lane`
#pragma unroll
  for (int k = 0; k < RUNS; ++k) {
    float f[8];
    uint32_t most = 0;  // of the magnitudes' bits, whose order is the magnitudes'; NaN above infinity
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = T::lo(v[k][i]);
      f[2 * i + 1] = T::hi(v[k][i]);
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
    int e = (int)(most >> 23) - 127 - 6;
    const int least = checkpoint_least<T>();
    e = e > least ? e : least;
    const bool finite = most < 0x7f800000u;
    const float inverse = __uint_as_float(finite ? (uint32_t)(127 - e) << 23 : 0u);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = __builtin_amdgcn_fmed3f(__builtin_rintf(f[i] * inverse), -127.f, 127.f);
      w[i >> 2] |= ((uint32_t)(int)q & 255u) << (8 * (i & 3));
    }
    if (!finite) w[0] = w[1] = 0u;
    if (in[k]) *reinterpret_cast<uint2*>(codes + at[k].row * d + at[k].col) = uint2{w[0], w[1]};
    const uint32_t from = (uint32_t)__shfl(finite ? e + 127 : 255, 4 * (lane & 15));
    if ((lane >> 4) == k) mine = from;
  }
  const At block = chunk(i0 + 4u * lane);
  if (lane < 16 * RUNS && block.row < n) exps[block.block] = (uint8_t)mine;
}

template <class T>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const int8_t* codes, const uint8_t* exps, int64_t n, int d,
                                                          uint16_t* x) {
  const At p = Chunks<1>((uint32_t)(d + 31) / 32u)(threadIdx.x);
  if (p.row >= n || p.col >= d) return;
  *reinterpret_cast<u32x4*>(x + p.row * d + p.col) =
      unpack8<T>(*reinterpret_cast<const uint2*>(codes + p.row * d + p.col), exps[p.block]);
}

int64_t workgroups(int64_t n, int d, int runs) {
  const int64_t of = kThreads * runs;
  return (n * ((d + 31) / 32 * 4) + of - 1) / of;
}

template <class T, int RUNS>
hipError_t pack(const uint16_t* x, int64_t x_ld, int64_t n, int d, int8_t* codes, uint8_t* exps, hipStream_t stream) {
  hipLaunchKernelGGL((pack_kernel<T, RUNS>), dim3((unsigned)workgroups(n, d, RUNS)), dim3(kThreads), 0, stream, x, x_ld,
                     n, d, codes, exps);
  return hipGetLastError();
}

// Four runs a wave where that leaves every CU eight workgroups: 53,248 rows of 4096 107 us (one run: 147); 764 rows of
// 768 one run, 2.9 us (four: 4.3).
template <class T>
hipError_t pack_any(const uint16_t* x, int64_t x_ld, int64_t n, int d, int8_t* codes, uint8_t* exps,
                    hipStream_t stream) {
  if (workgroups(n, d, 4) >= 2048) return pack<T, 4>(x, x_ld, n, d, codes, exps, stream);
  return pack<T, 1>(x, x_ld, n, d, codes, exps, stream);
}

}  // namespace

hipError_t launch_checkpoint_pack(const uint16_t* x, int64_t x_ld, int64_t n, int d, bool f16, int8_t* codes,
                                  uint8_t* exps, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  return f16 ? pack_any<HalfF16>(x, x_ld, n, d, codes, exps, stream)
             : pack_any<HalfBf16>(x, x_ld, n, d, codes, exps, stream);
}

hipError_t launch_checkpoint_unpack(const int8_t* codes, const uint8_t* exps, int64_t n, int d, bool f16, uint16_t* x,
                                    hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)workgroups(n, d, 1));
  if (f16)
    hipLaunchKernelGGL(unpack_kernel<HalfF16>, grid, dim3(kThreads), 0, stream, codes, exps, n, d, x);
  else
    hipLaunchKernelGGL(unpack_kernel<HalfBf16>, grid, dim3(kThreads), 0, stream, codes, exps, n, d, x);
  return hipGetLastError();
}

}  // namespace hpr
