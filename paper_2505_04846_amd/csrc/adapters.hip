// A shared projection with low-rank adapters of many requests beside it, and its gradients.
//
// Row t belongs to request s (off[s] <= t < off[s + 1]) with adapter a (negative: none):
//   h_t = scale_a A_a x_t            (rank values, rounded to 16 bits: see shrink_kernel)
//   y_t = W x_t + B_a h_t
// and for g_t = scale_a B_a^T dy_t:
//   dx_t = W^T dy_t + A_a^T g_t,   dA_a = sum_t g_t x_t^T,   dB_a = sum_t dy_t h_t^T.
// dx is the same operation on (dy, W^T, B^T, A^T), so the gradients run the forward's two kernels
// on transposed weights (transpose_kernel), and dA and dB are one kernel, outer_kernel, on (g, x)
// and (h, dy).
#include "common.h"
#include "half.h"
#include "kernels.h"
#include "tiles.h"

namespace hpr {

namespace {

__device__ __attribute__((aligned(16))) const uint32_t kZero16[4] = {0u, 0u, 0u, 0u};

// Bounds of request s, inside [0, n) whatever the offsets hold.
struct Rows {
  int64_t r0, r1;
};
__device__ __forceinline__ Rows rows_of(const AdapterArgs& a, int s) {
  auto clamp = [](int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); };
  Rows r;
  r.r0 = clamp(a.off[s], 0, a.n);
  r.r1 = clamp(a.off[s + 1], r.r0, a.n);
  return r;
}
// Adapter of request s, -1 for none (or one out of range).
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int s) {
  const int ad = a.adapter[s];
  return ad >= 0 && ad < a.n_ad ? ad : -1;
}

// ---- h ----------------------------------------------------------------------------------------

// h of 32 rows of one request.  The waves split k, each summing its part of the whole [rank, 32]
// block (rank on the rows of the product, so that a lane holds 4 consecutive values of its row's
// h), and join in LDS.  h is rounded to 16 bits once, with its scale: the operand of the product
// with B.  Its relative rounding reaches only the adapter's part of y.
constexpr int kShrinkRows = 32, kShrinkWaves = 4;

template <class T, int NB>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_kernel(AdapterArgs a, uint16_t* h) {
  __shared__ float part[kShrinkWaves][NB * 16][64];
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int s = find_seq(a.off, a.n_req, kShrinkRows, blockIdx.x);
  const Rows R = rows_of(a, s);
  const int64_t first = R.r0 + ((int64_t)blockIdx.x - (R.r0 / kShrinkRows + s)) * kShrinkRows;
  const int ad = adapter_of(a, s);
  if (first < R.r0 || first >= R.r1 || ad < 0) return;
  const int64_t t = first + col;
  const bool live = t < R.r1;
  const uint16_t* xr = a.x + (live ? t : R.r1 - 1) * (int64_t)a.k;
  const uint16_t* ar = a.a + (int64_t)ad * a.r * a.k;
  const uint16_t* arow[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int j = 32 * b + col;
    arow[b] = ar + (int64_t)(j < a.r ? j : a.r - 1) * a.k;
  }
  f32x16 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;
  const int steps = (a.k + 15) / 16;
  const int s0 = steps * wave / kShrinkWaves, s1 = steps * (wave + 1) / kShrinkWaves;
#pragma unroll 1
  for (int st = s0; st < s1; ++st) {
    const int d = 16 * st + 8 * half;
    const bool in = d < a.k;
    u32x4 xv = load16(xr + (in ? d : 0));
    if (!in) xv = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      u32x4 av = load16(arow[b] + (in ? d : 0));
      if (!in) av = u32x4{0u, 0u, 0u, 0u};
      acc[b] = T::mfma(av, xv, acc[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave][16 * b + r][lane] = acc[b][r];
  __syncthreads();
  const int rp = (a.r + 15) / 16 * 16;
  const float sc = a.scale[ad];
  // register groups of four: group g of NB * 4 holds ranks 32 (g / 4) + 8 (g % 4) + 4 half + 0..3
  for (int g = wave; g < NB * 4; g += kShrinkWaves) {
    const int j = 32 * (g >> 2) + 8 * (g & 3) + 4 * half;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kShrinkWaves; ++w) v[e] += part[w][4 * g + e][lane];
      v[e] = j + e < a.r ? v[e] * sc : 0.f;
    }
    if (live && j < rp)
      *reinterpret_cast<uint2*>(h + t * rp + j) = uint2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
  }
}

// ---- y ----------------------------------------------------------------------------------------

// Tile of BT rows of x by BM rows of W (columns of y), WT x WM waves, k in stages of 64 through
// two LDS stages.  W's rows are the rows of the product, so a lane holds 4 consecutive values of a
// row of y.  The adapters' part needs no LDS: for every run of rows of one request in the tile,
// h's rows (zero outside the run) and B's rows are read as operands.
template <class T, int BT, int BM, int WT, int WM>
__device__ __forceinline__ void expand_tile(const AdapterArgs& a, const uint16_t* __restrict__ h,
                                            uint16_t* __restrict__ y, int n_m) {
  constexpr int kW = WT * WM;
  constexpr int kTb = BT / 32 / WT, kMb = BM / 32 / WM;  // blocks per wave
  constexpr int kXBytes = BT * 128, kWBytes = BM * 128, kStage = kXBytes + kWBytes;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // 2 stages
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wave % WT, wm = wave / WT;
  const int64_t lin = xcd_linear(blockIdx.x, gridDim.x);
  const int64_t tt = lin / n_m;
  const int tm = (int)(lin - tt * n_m);
  const int64_t t0 = tt * BT;
  const int m0 = tm * BM;
  const int64_t left_t = a.n - t0;
  const int last_t = left_t < BT ? (int)left_t - 1 : BT - 1;
  const int last_m = a.m - m0 < BM ? a.m - m0 - 1 : BM - 1;

  const TileReads<64> rd(lane);
  const TileLoad<64, BT, kW> lx(wave, lane, 8);
  const TileLoad<64, BM, kW> lw(wave, lane, 8);
  const uint16_t* xb = a.x + t0 * a.k;
  const uint16_t* wb = a.w + (int64_t)m0 * a.k;
  const __amdgpu_buffer_rsrc_t rx = tile_rsrc(xb), rw = tile_rsrc(wb);
  int ox[lx.kLoads], ow[lw.kLoads];
#pragma unroll
  for (int j = 0; j < lx.kLoads; ++j)
    ox[j] = (lx.row[j] < last_t ? lx.row[j] : last_t) * a.k * 2 + lx.chunk[j];
#pragma unroll
  for (int j = 0; j < lw.kLoads; ++j)
    ow[j] = (lw.row[j] < last_m ? lw.row[j] : last_m) * a.k * 2 + lw.chunk[j];
  const int nk = (a.k + 63) / 64, nk_full = a.k / 64;
  auto issue = [&](int buf, int kk) {
    unsigned char* st = smem + buf * kStage;
    if (kk < nk_full) {
#pragma unroll
      for (int j = 0; j < lx.kLoads; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rx, (lds_void_t*)(st + (wave * lx.kLoads + j) * 1024), 16, ox[j], kk * 128, 0, 0);
#pragma unroll
      for (int j = 0; j < lw.kLoads; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rw, (lds_void_t*)(st + kXBytes + (wave * lw.kLoads + j) * 1024), 16, ow[j], kk * 128, 0, 0);
    } else if (kk < nk) {  // the end of k: chunks past it read zeros
#pragma unroll
      for (int j = 0; j < lx.kLoads; ++j) {
        const bool in = kk * 64 + lx.chunk[j] / 2 < a.k;
        const void* p = in ? (const void*)((const char*)xb + ox[j] + kk * 128) : (const void*)kZero16;
        __builtin_amdgcn_global_load_lds((glb_void_t*)p, (lds_void_t*)(st + (wave * lx.kLoads + j) * 1024),
                                         16, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < lw.kLoads; ++j) {
        const bool in = kk * 64 + lw.chunk[j] / 2 < a.k;
        const void* p = in ? (const void*)((const char*)wb + ow[j] + kk * 128) : (const void*)kZero16;
        __builtin_amdgcn_global_load_lds(
            (glb_void_t*)p, (lds_void_t*)(st + kXBytes + (wave * lw.kLoads + j) * 1024), 16, 0, 0);
      }
    }
  };

  f32x16 acc[kMb][kTb];
#pragma unroll
  for (int i = 0; i < kMb; ++i)
#pragma unroll
    for (int j = 0; j < kTb; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  issue(0, 0);
#pragma unroll 1
  for (int kk = 0; kk < nk; ++kk) {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    sync_lds();
    issue((kk + 1) & 1, kk + 1);
    const unsigned char* xs = smem + (kk & 1) * kStage;
    const unsigned char* ws = xs + kXBytes;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u32x4 fx[kTb], fw[kMb];
#pragma unroll
      for (int j = 0; j < kTb; ++j) fx[j] = rd.row_frag(xs, wt * kTb + j, s);
#pragma unroll
      for (int i = 0; i < kMb; ++i) fw[i] = rd.row_frag(ws, wm * kMb + i, s);
#pragma unroll
      for (int i = 0; i < kMb; ++i)
#pragma unroll
        for (int j = 0; j < kTb; ++j) acc[i][j] = T::mfma(fw[i], fx[j], acc[i][j]);
    }
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));

  // the adapters' part
  if (h && a.n_req > 0) {
    const int rp = (a.r + 15) / 16 * 16;
    const bool whole = a.r % 8 == 0;
    const int64_t wt0 = t0 + wt * kTb * 32;
    const int64_t wt1 = wt0 + kTb * 32 < a.n ? wt0 + kTb * 32 : a.n;
    int s = find_row(a.off, a.n_req, wt0);
#pragma unroll 1
    for (; s < a.n_req; ++s) {
      const Rows R = rows_of(a, s);
      if (R.r0 >= wt1) break;
      const int ad = adapter_of(a, s);
      if (R.r1 <= wt0 || R.r1 <= R.r0 || ad < 0) continue;
      const uint16_t* br = a.b + (int64_t)ad * a.m * a.r;
      auto b_frag = [&](int i, int d) {  // values [d, d + 8) of the lane's row of B, zero past r
        const int m = m0 + (wm * kMb + i) * 32 + col;
        const uint16_t* p = br + (int64_t)(m < a.m ? m : a.m - 1) * a.r;
        u32x4 f = {0u, 0u, 0u, 0u};
        if (whole) {
          if (d < a.r) f = load16(p + d);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (d + e < a.r) f[e >> 1] |= (uint32_t)p[d + e] << (16 * (e & 1));
        }
        return f;
      };
      auto h_frag = [&](int64_t t, int d) {
        u32x4 f = {0u, 0u, 0u, 0u};
        if (t >= R.r0 && t < R.r1) f = load16(h + t * rp + d);
        return f;
      };
      if (R.r0 <= wt0 && R.r1 >= wt1) {  // the run covers the wave's rows
#pragma unroll 1
        for (int d = 8 * half; d < rp; d += 16) {
          u32x4 fh[kTb], fb[kMb];
#pragma unroll
          for (int j = 0; j < kTb; ++j) fh[j] = h_frag(wt0 + 32 * j + col, d);
#pragma unroll
          for (int i = 0; i < kMb; ++i) fb[i] = b_frag(i, d);
#pragma unroll
          for (int i = 0; i < kMb; ++i)
#pragma unroll
            for (int j = 0; j < kTb; ++j) acc[i][j] = T::mfma(fb[i], fh[j], acc[i][j]);
        }
      } else {
        // rows outside the run keep their sums: a B that is not finite is none of theirs
#pragma unroll
        for (int j = 0; j < kTb; ++j) {
          const int64_t t = wt0 + 32 * j + col;
          if (R.r0 >= wt0 + 32 * j + 32 || R.r1 <= wt0 + 32 * j) continue;
          const bool in = t >= R.r0 && t < R.r1;
#pragma unroll
          for (int i = 0; i < kMb; ++i) {
            f32x16 v = acc[i][j];
#pragma unroll 1
            for (int d = 8 * half; d < rp; d += 16) v = T::mfma(b_frag(i, d), h_frag(t, d), v);
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = in ? v[r] : acc[i][j][r];
          }
        }
      }
    }
  }

#pragma unroll
  for (int j = 0; j < kTb; ++j) {
    const int64_t t = t0 + (wt * kTb + j) * 32 + col;
    if (t >= a.n) continue;
#pragma unroll
    for (int i = 0; i < kMb; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int m = m0 + (wm * kMb + i) * 32 + 8 * g + 4 * half;
        if (m < a.m)
          *reinterpret_cast<uint2*>(y + t * a.m + m) =
              uint2{T::pack(acc[i][j][4 * g], acc[i][j][4 * g + 1]),
                    T::pack(acc[i][j][4 * g + 2], acc[i][j][4 * g + 3])};
      }
  }
}

// (The body is a device function: the host pass knows no buffer resources.)
template <class T, int BT, int BM, int WT, int WM, int MINB>
__global__ __launch_bounds__(64 * WT * WM, MINB) void expand_kernel(AdapterArgs a, const uint16_t* h,
                                                                    uint16_t* y, int n_m) {
  expand_tile<T, BT, BM, WT, WM>(a, h, y, n_m);
}

// ---- transposed weights -----------------------------------------------------------------------

__global__ __launch_bounds__(256) void transpose_kernel(const uint16_t* in, uint16_t* out, int rows,
                                                        int cols) {
  __shared__ uint16_t tile[64][66];
  const int64_t base = (int64_t)blockIdx.z * rows * cols;
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  for (int i = y; i < 64; i += 4)
    if (r0 + i < rows && c0 + x < cols) tile[i][x] = in[base + (int64_t)(r0 + i) * cols + c0 + x];
  __syncthreads();
  for (int i = y; i < 64; i += 4)
    if (c0 + i < cols && r0 + x < rows) out[base + (int64_t)(c0 + i) * rows + r0 + x] = tile[x][i];
}

// ---- dA, dB -----------------------------------------------------------------------------------

// Partial sums over up to kOuterRows rows of one request: part[slot][j][c] = sum_t L[t,j] M[t,c],
// 64 ranks and 256 columns per workgroup, 64 columns per wave; rows in tiles of 64, both operands
// read by columns.
constexpr int kOuterRows = 512, kOuterWaves = 4;

template <class T>
__global__ __launch_bounds__(64 * kOuterWaves, 2) void outer_kernel(AdapterArgs a,
                                                                    const uint16_t* L,
                                                                    const uint16_t* M, int cols,
                                                                    int n_cb, float* part) {
  constexpr int kTile = 64 * 128;  // 64 rows of 64 values
  __shared__ __attribute__((aligned(1024))) unsigned char smem[(1 + kOuterWaves) * kTile];
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rp = (a.r + 15) / 16 * 16;
  const int n_jb = (rp + 63) / 64;
  const int cb = blockIdx.x % n_cb;
  const int jb = (int)(blockIdx.x / n_cb) % n_jb;
  const int64_t slot = blockIdx.x / n_cb / n_jb;
  const int s = find_seq(a.off, a.n_req, kOuterRows, slot);
  const Rows R = rows_of(a, s);
  const int64_t first = R.r0 + (slot - (R.r0 / kOuterRows + s)) * kOuterRows;
  if (first < R.r0 || first >= R.r1 || adapter_of(a, s) < 0) return;
  const int64_t end = R.r1 < first + kOuterRows ? R.r1 : first + kOuterRows;

  const int c0 = cb * 64 * kOuterWaves + wave * 64;
  const int j0 = jb * 64;
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const TileReads<64> rd(lane);
  const int lr = lane >> 3;  // row of a wave load, 8 rows of 8 chunks
#pragma unroll 1
  for (int64_t t = first; t < end; t += 64) {
    sync_lds();
    // rows past the end are zero in both tiles; columns past the last repeat it, and their sums are
    // not stored
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 8 * j + lr;
      const int c = (lane & 7) ^ swz<64>(r);
      const bool in = t + r < end;
      int cc = c0 + 8 * c;
      if (cc >= cols) cc = cols - 8;
      const void* p = in ? (const void*)(M + (t + r) * cols + cc) : (const void*)kZero16;
      load_lds16(p, LDS_ADDRESS(smem) + (1 + wave) * kTile + j * 1024);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = 8 * (2 * wave + j) + lr;
      const int c = (lane & 7) ^ swz<64>(r);
      const bool in = t + r < end;
      int cc = j0 + 8 * c;
      if (cc >= rp) cc = rp - 8;
      const void* p = in ? (const void*)(L + (t + r) * rp + cc) : (const void*)kZero16;
      load_lds16(p, LDS_ADDRESS(smem) + (2 * wave + j) * 1024);
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    sync_lds();
    const unsigned char* ms = smem + (1 + wave) * kTile;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        u32x4 fm[2], fl[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fm[i] = rd.tr_frag(ms, b, st, i);
          fl[i] = rd.tr_frag(smem, b, st, i);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = T::mfma(fm[i], fl[j], acc[i][j]);
      }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int jj = j0 + 32 * j + col;
    if (jj >= rp) continue;
    float* dst = part + (slot * rp + jj) * (int64_t)cols;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = c0 + 32 * i + 8 * g + 4 * half;
        if (c < cols)
          *reinterpret_cast<f32x4*>(dst + c) = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1],
                                                     acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
      }
  }
}

// out[ad] = the sum of its requests' parts, in their order.  A thread per (j, c).
template <class T>
__global__ __launch_bounds__(256) void outer_join_kernel(AdapterArgs a, int cols, int transposed,
                                                         const float* part, uint16_t* out) {
  const int ad = blockIdx.y;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(i / cols), c = (int)(i - (int64_t)j * cols);
  if (j >= a.r) return;
  const int rp = (a.r + 15) / 16 * 16;
  float sum = 0.f;
  for (int s = 0; s < a.n_req; ++s) {
    if (adapter_of(a, s) != ad) continue;
    const Rows R = rows_of(a, s);
    const int64_t slot0 = R.r0 / kOuterRows + s;
    const int64_t n = (R.r1 - R.r0 + kOuterRows - 1) / kOuterRows;
    for (int64_t k = 0; k < n; ++k) sum += part[((slot0 + k) * rp + j) * (int64_t)cols + c];
  }
  const uint16_t v = (uint16_t)T::pack(sum, 0.f);
  if (transposed)
    out[((int64_t)ad * cols + c) * a.r + j] = v;
  else
    out[((int64_t)ad * a.r + j) * cols + c] = v;
}

template <class T>
hipError_t shrink(const AdapterArgs& a, uint16_t* h, hipStream_t s) {
  const int64_t grid = a.n / kShrinkRows + a.n_req;
  const int nb = (a.r + 31) / 32;
  if (nb == 1)
    hipLaunchKernelGGL((shrink_kernel<T, 1>), dim3((unsigned)grid), dim3(64 * kShrinkWaves), 0, s, a, h);
  else if (nb == 2)
    hipLaunchKernelGGL((shrink_kernel<T, 2>), dim3((unsigned)grid), dim3(64 * kShrinkWaves), 0, s, a, h);
  else
    hipLaunchKernelGGL((shrink_kernel<T, 4>), dim3((unsigned)grid), dim3(64 * kShrinkWaves), 0, s, a, h);
  return hipGetLastError();
}

template <class T, int BT, int BM, int WT, int WM, int MINB>
hipError_t expand_as(const AdapterArgs& a, const uint16_t* h, uint16_t* y, hipStream_t s) {
  const int n_m = (a.m + BM - 1) / BM;
  const int64_t grid = (a.n + BT - 1) / BT * n_m;
  constexpr int lds = 2 * (BT + BM) * 128;
  if (lds > 65536) {  // beyond the default dynamic LDS limit
    const void* fn = (const void*)expand_kernel<T, BT, BM, WT, WM, MINB>;
    const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((expand_kernel<T, BT, BM, WT, WM, MINB>), dim3((unsigned)grid),
                     dim3(64 * WT * WM), lds, s, a, h, y, n_m);
  return hipGetLastError();
}

template <class T>
hipError_t expand(const AdapterArgs& a, const uint16_t* h, uint16_t* y, hipStream_t s) {
  const int64_t tiles = ((a.n + 255) / 256) * ((a.m + 255) / 256);
  if (tiles >= 128) return expand_as<T, 256, 256, 4, 2, 1>(a, h, y, s);
  if (a.n > 64) return expand_as<T, 128, 128, 2, 2, 2>(a, h, y, s);
  return expand_as<T, 32, 64, 1, 2, 2>(a, h, y, s);
}

template <class T>
hipError_t outer(const AdapterArgs& a, const uint16_t* L, const uint16_t* M, int cols, bool transposed,
                 float* part, uint16_t* out, hipStream_t s) {
  const int rp = adapter_rank_pad(a.r);
  const int n_cb = (cols + 64 * kOuterWaves - 1) / (64 * kOuterWaves), n_jb = (rp + 63) / 64;
  const int64_t grid = adapter_outer_parts(a.n, a.n_req) * n_cb * n_jb;
  if (grid > 0)
    hipLaunchKernelGGL((outer_kernel<T>), dim3((unsigned)grid), dim3(64 * kOuterWaves), 0, s, a, L, M,
                       cols, n_cb, part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t each = ((int64_t)a.r * cols + 255) / 256;
  hipLaunchKernelGGL((outer_join_kernel<T>), dim3((unsigned)each, (unsigned)a.n_ad), dim3(256), 0, s, a,
                     cols, transposed ? 1 : 0, part, out);
  return hipGetLastError();
}

}  // namespace

int64_t adapter_outer_parts(int64_t n, int n_req) { return n / kOuterRows + n_req; }

hipError_t launch_adapter_shrink(const AdapterArgs& a, uint16_t* h, hipStream_t stream) {
  if (a.n == 0 || a.n_req == 0) return hipSuccess;
  return a.f16 ? shrink<HalfF16>(a, h, stream) : shrink<HalfBf16>(a, h, stream);
}

hipError_t launch_adapter_expand(const AdapterArgs& a, const uint16_t* h, uint16_t* y,
                                 hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  return a.f16 ? expand<HalfF16>(a, h, y, stream) : expand<HalfBf16>(a, h, y, stream);
}

hipError_t launch_transpose(const uint16_t* in, uint16_t* out, int64_t count, int rows, int cols,
                            hipStream_t stream) {
  if (count == 0) return hipSuccess;
  hipLaunchKernelGGL(transpose_kernel,
                     dim3((unsigned)((cols + 63) / 64), (unsigned)((rows + 63) / 64), (unsigned)count),
                     dim3(256), 0, stream, in, out, rows, cols);
  return hipGetLastError();
}

hipError_t launch_adapter_outer(const AdapterArgs& a, const uint16_t* L, const uint16_t* M, int cols,
                                bool transposed, float* part, uint16_t* out, hipStream_t stream) {
  if (a.n_ad == 0) return hipSuccess;
  return a.f16 ? outer<HalfF16>(a, L, M, cols, transposed, part, out, stream)
               : outer<HalfBf16>(a, L, M, cols, transposed, part, out, stream);
}

}  // namespace hpr
