// A shared projection with low-rank adapters of many requests beside it, and its gradients.
//
// Row t belongs to request s (off[s] <= t < off[s + 1]) with adapter a (negative: none):
//   h_t = scale_a A_a x_t            (rank values, rounded to 16 bits: see shrink_kernel)
//   y_t = W x_t + B_a h_t
// and for g_t = scale_a B_a^T dy_t:
//   dx_t = W^T dy_t + A_a^T g_t,   dA_a = sum_t g_t x_t^T,   dB_a = sum_t dy_t h_t^T.
// dx is the same operation on (dy, W^T, B^T, A^T), so the gradients run the forward's two kernels
// on transposed weights (prepare_kernel), and dA and dB are one kernel, outer_kernel, on (g, x)
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
__device__ __forceinline__ Rows rows_of(const int64_t* off, int64_t n, int s) {
  auto clamp = [](int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); };
  Rows r;
  r.r0 = clamp(off[s], 0, n);
  r.r1 = clamp(off[s + 1], r.r0, n);
  return r;
}
__device__ __forceinline__ Rows rows_of(const AdapterArgs& a, int s) { return rows_of(a.off, a.n, s); }
// Adapter of request s, -1 for none (or one out of range).
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int s) {
  const int ad = a.adapter[s];
  return ad >= 0 && ad < a.n_ad ? ad : -1;
}

// ---- a wave's own product ----------------------------------------------------------------------

// acc[b][c] = rows [32 b, 32 b + 32) of P times rows [32 c, + 32) of X, over stages [kk0, kk1) of 64 values,
// by one wave: its NST LDS stages are its own, so waves that split k run without a barrier.  Whole 128-byte
// lines go straight to LDS (operands read from memory by lanes touch twice as many lines a load: a token's
// projection took 22 us that way).  Of P, ROWS rows are loaded; the results of the rest of its last 32 are
// not to be used (their operands are what LDS holds past the stage, of this wave's or another's).
template <class T, int NB, int XB, int NST = 2, int ROWS = 32 * NB>
struct WaveProduct {
  static constexpr int kStage = XB * 4096 + ROWS * 128;
  static constexpr int kBytes = NST * kStage;
  static constexpr int kPast = (32 * NB - ROWS) * 128;  // LDS read past the stages
  static constexpr int kX = 4 * XB, kLoads = 4 * XB + ROWS / 8;
  // x, p: first rows; x_last, p_last: their last valid row, which the rows past it repeat
  static __device__ __forceinline__ void run(const uint16_t* x, int x_last, const uint16_t* p, int p_last,
                                             int k, int kk0, int kk1, unsigned char* lds, int lane,
                                             f32x16 (&acc)[NB][XB]) {
    const __amdgpu_buffer_rsrc_t rx = tile_rsrc(x), rp = tile_rsrc(p);
    const TileReads<64> rd(lane);
    int off[kLoads], chunk[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = 8 * (j < kX ? j : j - kX) + (lane >> 3);
      const int last = j < kX ? x_last : p_last;
      chunk[j] = ((lane & 7) ^ swz<64>(r)) * 8;
      off[j] = (r < last ? r : last) * k * 2 + chunk[j] * 2;
    }
    const int whole = k / 64;
    auto issue = [&](int buf, int kk) {
      unsigned char* st = lds + buf * kStage;
      if (kk < whole) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(j < kX ? rx : rp, (lds_void_t*)(st + j * 1024), 16,
                                                   off[j], kk * 128, 0, 0);
      } else {  // the end of k: chunks past it read zeros
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const char* src = (const char*)(j < kX ? x : p) + off[j] + kk * 128;
          const void* from = kk * 64 + chunk[j] < k ? (const void*)src : (const void*)kZero16;
          __builtin_amdgcn_global_load_lds((glb_void_t*)from, (lds_void_t*)(st + j * 1024), 16, 0, 0);
        }
      }
    };
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int c = 0; c < XB; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][c][r] = 0.f;
    static_assert(NST == 2 || NST == 3, "the waits below");
    if (kk0 < kk1) issue(0, kk0);
    if (NST == 3 && kk0 + 1 < kk1) issue(1, kk0 + 1);
#pragma unroll 1
    for (int kk = kk0, buf = 0; kk < kk1; ++kk, buf = buf + 1 < NST ? buf + 1 : 0) {
      if (kk + NST - 1 < kk1) {
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);  // that stage's reads are done
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        issue(buf > 0 ? buf - 1 : NST - 1, kk + NST - 1);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 1) * kLoads));
      } else if (NST == 3 && kk + 1 < kk1) {
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(kLoads));
      } else {
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
      }
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      const unsigned char* st = lds + buf * kStage;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        u32x4 fx[XB];
#pragma unroll
        for (int c = 0; c < XB; ++c) fx[c] = rd.row_frag(st, c, s);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const u32x4 fp = rd.row_frag(st + XB * 4096, b, s);
#pragma unroll
          for (int c = 0; c < XB; ++c) acc[b][c] = T::mfma(fp, fx[c], acc[b][c]);
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
  }
};

// ---- h ----------------------------------------------------------------------------------------

// h of 32 XB rows of one request, 32 NB ranks.  W waves split k, each summing its part of the [32 NB, 32 XB]
// block (rank on the rows of the product, so that a lane holds 4 consecutive values of its row's
// h), and join in LDS.  h is rounded to 16 bits once, with its scale: the operand of the product
// with B.  Its relative rounding reaches only the adapter's part of y.  Bound by x: 13,063 rows of 4096
// of 64 requests, rank 16, 20 us (107 MB, 5.3 TB/s out of the caches); 32 rows of 32 requests 8 us, a
// wave's eight waits for memory.
//
// fp16 has no bits below 2^-24 and few below 2^-14, where g lies while B is near its start at zero and dy is small,
// and h where A or x is.  The gradients of A and B, in which nothing else covers that loss, read g and h in
// two numbers (LOW): the value's rounding and, below 1 (above, the rounding alone keeps 11 bits), the rest of it
// times 2^24, exactly apart.  4096 rows, B and dy of 1e-4: dA was off by 2.7e-2, as rounding g alone makes it.
// y and dx read the roundings alone: what they lose there, at most 2^-25 a rank, is of the size of what their own
// rounding loses.  Forward and gradients in fp16, us with it (without): 13,057 rows, 4096 -> 4096, rank 64 1,006
// (937: h again, x and dy read twice for 64 ranks), 4,000 rows, 768 -> 768, rank 16 60 (54), 764 rows, 768 -> 2304,
// rank 8 53 (52).
constexpr float kRest = 0x1p24f;
__device__ __forceinline__ float rest(float v, float rounded) {
  return __builtin_fabsf(v) < 1.f ? (v - rounded) * kRest : 0.f;
}

template <class T, int NB, int XB, int W>
__device__ __forceinline__ void shrink_tile(const AdapterArgs& a, uint16_t* h, uint16_t* low) {
  using P = WaveProduct<T, NB, XB>;
  constexpr int kRows = 32 * XB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // W * P::kBytes
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int s = find_seq(a.off, a.n_req, kRows, blockIdx.x);
  const Rows R = rows_of(a, s);
  const int64_t first = R.r0 + ((int64_t)blockIdx.x - ((uint32_t)R.r0 / kRows + (uint32_t)s)) * kRows;
  const int ad = adapter_of(a, s);
  if (first < R.r0 || first >= R.r1 || ad < 0) return;
  const int last = R.r1 - first < kRows ? (int)(R.r1 - first) - 1 : kRows - 1;
  const int nk = (a.k + 63) / 64;
  const int j0 = blockIdx.y * 32 * NB, left = a.r - j0;  // ranks
  f32x16 acc[NB][XB];
  unsigned char* own = smem + wave * P::kBytes;
  P::run(a.x + first * a.k, last, a.a + ((int64_t)ad * a.r + j0) * a.k,
         left < 32 * NB ? left - 1 : 32 * NB - 1, a.k, nk * wave / W, nk * (wave + 1) / W, own, lane, acc);
  float* part = reinterpret_cast<float*>(own);  // [NB * XB * 16][64]
  static_assert(NB * XB * 4096 <= P::kBytes, "the wave's sums fit its stages");
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int c = 0; c < XB; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) part[(16 * (b * XB + c) + r) * 64 + lane] = acc[b][c][r];
  __syncthreads();
  const int rp = (a.r + 15) / 16 * 16;
  const float sc = a.scale[ad];
  // register groups of four: group g of block (b, c) holds ranks j0 + 32 b + 8 g + 4 half + 0..3 of row
  // 32 c + col
  for (int i = wave; i < NB * XB * 4; i += W) {
    const int bc = i >> 2, j = j0 + 32 * (bc / XB) + 8 * (i & 3) + 4 * half, t = 32 * (bc % XB) + col;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w)
        v[e] += reinterpret_cast<const float*>(smem + w * P::kBytes)[(4 * i + e) * 64 + lane];
      v[e] = j + e < a.r ? v[e] * sc : 0.f;
    }
    if (t <= last && j < rp) {
      const uint2 w = {T::pack(v[0], v[1]), T::pack(v[2], v[3])};
      *reinterpret_cast<uint2*>(h + (first + t) * rp + j) = w;
      if constexpr (T::kNarrow)
        if (low)
          *reinterpret_cast<uint2*>(low + (first + t) * rp + j) =
              uint2{T::pack(rest(v[0], T::lo(w.x)), rest(v[1], T::hi(w.x))),
                    T::pack(rest(v[2], T::lo(w.y)), rest(v[3], T::hi(w.y)))};
    }
  }
}

struct ShrinkArgs {
  ShrinkJob job[2];
};

// (The bodies are device functions: the host pass knows no buffer resources.)
template <class T, int NB, int XB, int W>
__global__ __launch_bounds__(64 * W) void shrink_kernel(ShrinkArgs p) {
  const ShrinkJob& q = p.job[blockIdx.z];
  shrink_tile<T, NB, XB, W>(q.a, q.h, q.low);
}

// ---- y ----------------------------------------------------------------------------------------

// Tile of BT rows of x by BM rows of W (columns of y), WT x WM waves, k in stages of 64 through NST LDS
// stages.  W's rows are the rows of the product, so a lane holds 4 consecutive values of a row of y.
//
// Measured: 13,063 rows, 4096 -> 6144 (256 x 256 tiles) 505-590 us from card to card, 1.11-1.30 PFLOP/s,
// where the library's product of 12,960 rows alone takes 584-588 us; 13,057 rows, 4096 -> 4096 340-370 us and 40 us
// for its last round in 128 x 128 tiles, 1.07-1.15 PFLOP/s (library 332-343 us).  The matrix cores are busy 65-70 %
// of the cycles; on random operands the card's power limit then holds the clock at 1.6-1.8 GHz.  764 rows, 768 -> 2304 (64 x 64) 11 us: launch
// and the waits for the request, its h and its B, then 12 stages at 0.17 us.
//
// The adapters' part comes first, while the first stage is on its way, and needs no LDS: for every run of
// rows of one request in the wave's rows, h's rows and B's rows are read as operands, and the product
// goes to the rows of the run alone (a B that is not finite is not another request's).
template <class T, int BT, int BM, int WT, int WM, int NST>
__device__ __forceinline__ void expand_tile(const AdapterArgs& a, const uint16_t* __restrict__ h,
                                            uint16_t* __restrict__ y, int n_m) {
  constexpr int kW = WT * WM;
  constexpr int kTb = BT / 32 / WT, kMb = BM / 32 / WM;  // blocks per wave
  constexpr int kXBytes = BT * 128, kWBytes = BM * 128, kStage = kXBytes + kWBytes;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // NST stages
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wt = wave % WT, wm = wave / WT;
  // An XCD walks a contiguous run of tiles, four row tiles abreast: the tiles that it holds at a time
  // (32 of the widest) read 4 row tiles and 8 column tiles, not 1 or 2 and all the columns.
  const uint32_t lin = (uint32_t)xcd_linear(blockIdx.x, gridDim.x);
  const uint32_t n_t = (uint32_t)((a.n - a.row0 + BT - 1) / BT);
  const uint32_t g0 = lin / (4u * n_m) * 4u, in_g = lin - g0 * n_m;
  const uint32_t abreast = n_t - g0 < 4u ? n_t - g0 : 4u;
  const int tm = (int)(in_g / abreast);
  const int64_t t0 = a.row0 + (int64_t)(g0 + in_g % abreast) * BT;
  const int m0 = tm * BM;
  const int64_t left_t = a.n - t0;
  const int last_t = left_t < BT ? (int)left_t - 1 : BT - 1;
  const int last_m = a.m - m0 < BM ? a.m - m0 - 1 : BM - 1;

  const TileReads<64> rd(lane);
  const TileLoad<64, BT, kW> lx(wave, lane, 8);
  const TileLoad<64, BM, kW> lw(wave, lane, 8);
  constexpr int kLoads = lx.kLoads + lw.kLoads;
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
  // Stage kk into ring buffer buf.  Chunks past the end of k read zeros, so past the last stage too
  // (the ring keeps its number of loads in flight).
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
    } else {
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
  // A wave of one block reads a whole stage's operands ahead of its products, and so hands the stage back
  // when the next is begun (4096 -> 14336, 146 rows: 51 -> 46 us of the call); the others keep the stage
  // that they compute on.
  constexpr bool kAhead = kMb * kTb == 1;
#pragma unroll
  for (int s = 0; s < (kAhead ? NST : NST - 1); ++s) issue(s, s);

  f32x16 acc[kMb][kTb];
#pragma unroll
  for (int i = 0; i < kMb; ++i)
#pragma unroll
    for (int j = 0; j < kTb; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // the adapters' part: a lane looks at one request of the wave's rows, 64 at a time
  if (h && a.n_req > 0) {
    const int rp = (a.r + 15) / 16 * 16;
    const bool whole = a.r % 8 == 0;
    const int64_t w0 = t0 + wt * kTb * 32;
#pragma unroll 1
    for (int base = find_row(a.off, a.n_req, w0); base < a.n_req; base += 64) {
      const int s = base + lane < a.n_req ? base + lane : a.n_req - 1;
      const Rows R = rows_of(a, s);
      const int ad = adapter_of(a, s);
      auto in_wave = [&](int64_t r) { return (int)(r < w0 ? 0 : (r - w0 < 32 * kTb ? r - w0 : 32 * kTb)); };
      const int lo = in_wave(R.r0), hi = in_wave(R.r1);
      const unsigned long long runs = __ballot(base + lane < a.n_req && lo < hi && ad >= 0);
#pragma unroll
      for (int j = 0; j < kTb; ++j) {
        const int row = 32 * j + col;
#pragma unroll 1
        for (unsigned long long left = runs & __ballot(lo < 32 * j + 32 && hi > 32 * j); left; left &= left - 1) {
          const int i = __builtin_ctzll(left);
          const int r_lo = __builtin_amdgcn_readlane(lo, i), r_hi = __builtin_amdgcn_readlane(hi, i);
          const uint16_t* br = a.b + (int64_t)__builtin_amdgcn_readlane(ad, i) * a.m * a.r;
          const bool in = row >= r_lo && row < r_hi;
          f32x16 v[kMb];
#pragma unroll
          for (int i = 0; i < kMb; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) v[i][r] = 0.f;
#pragma unroll 1
          for (int d = 8 * half; d < rp; d += 16) {
            u32x4 fh = {0u, 0u, 0u, 0u};
            if (in) fh = load16(h + (w0 + row) * rp + d);
#pragma unroll
            for (int i = 0; i < kMb; ++i) {
              const int m = m0 + (wm * kMb + i) * 32 + col;
              const uint16_t* p = br + (int64_t)(m < a.m ? m : a.m - 1) * a.r;
              u32x4 fb = {0u, 0u, 0u, 0u};
              if (whole) {
                if (d < a.r) fb = load16(p + d);
              } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (d + e < a.r) fb[e >> 1] |= (uint32_t)p[d + e] << (16 * (e & 1));
              }
              v[i] = T::mfma(fb, fh, v[i]);
            }
          }
#pragma unroll
          for (int i = 0; i < kMb; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = in ? v[i][r] : acc[i][j][r];
        }
      }
      if (__any(R.r0 >= w0 + 32 * kTb)) break;
    }
  }

  struct Frags {
    u32x4 x[kTb], w[kMb];
  };
  auto read_frags = [&](int buf, int s, Frags& f) {
    const unsigned char* xs = smem + buf * kStage;
#pragma unroll
    for (int j = 0; j < kTb; ++j) f.x[j] = rd.row_frag(xs, wt * kTb + j, s);
#pragma unroll
    for (int i = 0; i < kMb; ++i) f.w[i] = rd.row_frag(xs + kXBytes, wm * kMb + i, s);
  };
  auto mfma = [&](const Frags& f) {
#pragma unroll
    for (int i = 0; i < kMb; ++i)
#pragma unroll
      for (int j = 0; j < kTb; ++j) acc[i][j] = T::mfma(f.w[i], f.x[j], acc[i][j]);
  };
  if constexpr (kAhead) {
    Frags f[2][4];
    auto stage = [&](int buf, int kk, Frags (&now)[4], Frags (&then)[4]) {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 2) * kLoads));
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      sync_lds();  // the next stage has landed, and nobody reads this one any more
      issue(buf, kk + NST);
      const int nxt = buf + 1 < NST ? buf + 1 : 0;
#pragma unroll
      for (int s = 0; s < 4; ++s) read_frags(nxt, s, then[s]);  // (past the last stage: zeros, not used)
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < 4; ++s) mfma(now[s]);
      return nxt;
    };
    __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 1) * kLoads));
    sync_lds();
#pragma unroll
    for (int s = 0; s < 4; ++s) read_frags(0, s, f[0][s]);
    int buf = 0;
#pragma unroll 1
    for (int kk = 0; kk < nk; kk += 2) {
      buf = stage(buf, kk, f[0], f[1]);
      if (kk + 1 < nk) buf = stage(buf, kk + 1, f[1], f[0]);
    }
  } else {
    // The stages of the ring: NST - 1 are in flight when one is computed on.  One barrier per stage,
    // before its last k-step, whose products run while the next stage's first operands are read.
    Frags f0, f1;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 2) * kLoads));
    sync_lds();
    read_frags(0, 0, f0);
#pragma unroll 1
    for (int kk = 0, buf = 0; kk < nk; ++kk) {
      const int nxt = buf + 1 < NST ? buf + 1 : 0, free_ = buf > 0 ? buf - 1 : NST - 1;
      issue(free_, kk + NST - 1);
      __builtin_amdgcn_sched_barrier(0);
      read_frags(buf, 1, f1);
      mfma(f0);
      read_frags(buf, 2, f0);
      mfma(f1);
      read_frags(buf, 3, f1);
      mfma(f0);
      // each k-step's products alternate with the reads of the next one's operands
#pragma unroll
      for (int u = 0; u < 3; ++u) {
#pragma unroll
        for (int t = 0; t < kMb * kTb; ++t) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          if (t < kTb + kMb) __builtin_amdgcn_sched_group_barrier(0x100, kMb * kTb >= kTb + kMb ? 1 : kTb + kMb, 0);
        }
      }
      __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 2) * kLoads));
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      sync_lds();
      read_frags(nxt, 0, f0);  // (past the last stage: zeros, or rows that are read by nobody)
      __builtin_amdgcn_sched_barrier(0);
      mfma(f1);
      buf = nxt;
    }
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // no load may still target LDS when it is reused or ends

  // y through LDS, so that memory sees whole rows: a wave's 32 kTb rows of 32 kMb values, one 32-row
  // block at a time
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  sync_lds();
  constexpr int kRow = 64 * kMb;                                // bytes of a wave's row
  static_assert(kW * 32 * kRow <= NST * kStage, "the waves' blocks fit the ring");
  unsigned char* own = smem + wave * 32 * kRow;
  constexpr int kCh = kRow / 16, kPer = 64 / kCh;               // chunks of a row, rows of a wave store
  const int mw = m0 + wm * kMb * 32;
#pragma unroll
  for (int j = 0; j < kTb; ++j) {
    const int64_t r0 = t0 + (wt * kTb + j) * 32;
    __atomic_signal_fence(__ATOMIC_SEQ_CST);  // (a wave's LDS operations execute in program order)
#pragma unroll
    for (int i = 0; i < kMb; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(own + col * kRow + (((4 * i + g) ^ (col % kCh)) << 4) + 8 * half) =
            uint2{T::pack(acc[i][j][4 * g], acc[i][j][4 * g + 1]),
                  T::pack(acc[i][j][4 * g + 2], acc[i][j][4 * g + 3])};
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    uint16_t* dst = y + r0 * a.m + mw;
#pragma unroll
    for (int k = 0; k < 32 / kPer; ++k) {
      const int r = k * kPer + lane / kCh, c = (lane % kCh) ^ (r % kCh);
      const u32x4 v = *reinterpret_cast<const u32x4*>(own + r * kRow + (lane % kCh) * 16);
      if (r0 + r < a.n && mw + 8 * c < a.m) *reinterpret_cast<u32x4*>(dst + (int64_t)r * a.m + 8 * c) = v;
    }
  }
}

template <class T, int BT, int BM, int WT, int WM, int NST, int MINB>
__global__ __launch_bounds__(64 * WT * WM, MINB) void expand_kernel(AdapterArgs a, const uint16_t* h,
                                                                    uint16_t* y, int n_m) {
  expand_tile<T, BT, BM, WT, WM, NST>(a, h, y, n_m);
}

// Few rows: 32 rows of x by BM = 32 or 16 rows of W per workgroup.  Eight waves split k; meanwhile the
// threads of BM / 4 others form the adapter's part of two values of y each, from their row's own h and B,
// and add the eight sums to it in the end.  32 rows of 32 requests, 4096 -> 4096: 8.8 us, 3.8 TB/s of W; what
// is left is the launch and four waits for memory.
constexpr int kFewWaves = 8;
template <class T, int BM>
using FewProduct = WaveProduct<T, 1, 1, BM == 32 ? 2 : 3, BM>;
template <class T, int BM>
constexpr int kFewLds = kFewWaves * FewProduct<T, BM>::kBytes + FewProduct<T, BM>::kPast;
template <int BM>
constexpr int kFewThreads = 64 * (kFewWaves + BM / 4);

// Two values of B h of row t, columns m and m + 1.
template <class T>
__device__ __forceinline__ float2 adapter_part(const AdapterArgs& a, const uint16_t* h, int64_t t, int m) {
  float2 v = {0.f, 0.f};
  if (a.n_req == 0 || t >= a.n || m >= a.m) return v;
  // the row's request (the last that starts at or before it)
  int lo = 0, n = a.n_req;
  while (n > 1) {
    const int step = n / 2;
    if (a.off[lo + step] <= t) lo += step, n -= step;
    else n = step;
  }
  const int ad = adapter_of(a, lo);
  if (ad < 0 || a.off[lo] > t || t >= a.off[lo + 1]) return v;
  const uint16_t* hr = h + t * ((a.r + 15) / 16 * 16);
  const uint16_t* b0 = a.b + ((int64_t)ad * a.m + m) * a.r;
  if (a.r % 8 == 0) {
    for (int d = 0; d < a.r; d += 8) {
      const u32x4 hv = load16(hr + d), u = load16(b0 + d), w = load16(b0 + a.r + d);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v.x += T::lo(hv[q]) * T::lo(u[q]) + T::hi(hv[q]) * T::hi(u[q]);
        v.y += T::lo(hv[q]) * T::lo(w[q]) + T::hi(hv[q]) * T::hi(w[q]);
      }
    }
  } else {
    for (int d = 0; d < a.r; ++d) {
      v.x += T::lo(hr[d]) * T::lo(b0[d]);
      v.y += T::lo(hr[d]) * T::lo(b0[a.r + d]);
    }
  }
  return v;
}

template <class T, int BM>
__device__ __forceinline__ void expand_few(const AdapterArgs& a, const uint16_t* h, uint16_t* y, int n_m) {
  using P = FewProduct<T, BM>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // kFewLds
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = (int)(blockIdx.x % (uint32_t)n_m) * BM;
  const int64_t t0 = (int64_t)(blockIdx.x / (uint32_t)n_m) * 32;
  if (wave < kFewWaves) {
    const int nk = (a.k + 63) / 64;
    f32x16 acc[1][1];
    unsigned char* own = smem + wave * P::kBytes;
    P::run(a.x + t0 * a.k, a.n - t0 < 32 ? (int)(a.n - t0) - 1 : 31, a.w + (int64_t)m0 * a.k,
           a.m - m0 < BM ? a.m - m0 - 1 : BM - 1, a.k, nk * wave / kFewWaves, nk * (wave + 1) / kFewWaves, own,
           lane, acc);
    float* part = reinterpret_cast<float*>(own);  // [16][64]
#pragma unroll
    for (int r = 0; r < 16; ++r) part[r * 64 + lane] = acc[0][0][r];
    __syncthreads();
    return;
  }
  // thread: two columns of a row: entries e, e + 1 of lane (row, half) with column = 8 (e / 4) + 4 half + e % 4
  const int i = threadIdx.x - 64 * kFewWaves, row = i / (BM / 2), m = 2 * (i % (BM / 2));
  const int64_t t = t0 + row;
  float2 v = adapter_part<T>(a, h, t, m0 + m);
  __syncthreads();
  const int e = 4 * (m >> 3) + (m & 3), at = row + 32 * ((m >> 2) & 1);
  float2 w = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kFewWaves; ++k) {
    const float* from = reinterpret_cast<const float*>(smem + k * P::kBytes);
    w.x += from[e * 64 + at];
    w.y += from[(e + 1) * 64 + at];
  }
  if (t < a.n && m0 + m < a.m) *reinterpret_cast<uint32_t*>(y + t * a.m + m0 + m) = T::pack(w.x + v.x, w.y + v.y);
}

template <class T, int BM>
__global__ __launch_bounds__(kFewThreads<BM>) void expand_few_kernel(AdapterArgs a, const uint16_t* h,
                                                                     uint16_t* y, int n_m) {
  expand_few<T, BM>(a, h, y, n_m);
}

// ---- rows by adapter --------------------------------------------------------------------------

// A workgroup for kOrderAdapters adapters: counts their rows, places every request of theirs behind the
// earlier ones of its adapter, and writes down its rows.  Four waves take a run of requests each, 64 at a
// time.  The only atomics add integers, whose sum has no order.  (Whatever the offsets hold, nothing is
// written past n; what then stays unwritten is clamped where it is read.)
constexpr int kOrderAdapters = 256;
constexpr int kOrderLds = 4 * kOrderAdapters + 8;  // words

__device__ __forceinline__ void order_rows(const AdapterArgs& a, const AdapterOrder& to, uint32_t* lds, int a0) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t* sums = lds + 4 * kOrderAdapters;
  uint32_t* count = lds + wave * kOrderAdapters;  // rows of the wave's requests, then where the next ones go
#pragma unroll
  for (int w = 0; w < 4; ++w) lds[w * kOrderAdapters + threadIdx.x] = 0;
  __syncthreads();
  const int64_t chunks = (a.n_req + 63) / 64;
  const int c0 = (int)(chunks * wave / 4), c1 = (int)(chunks * (wave + 1) / 4);
  struct Request {
    int first;
    uint32_t rows;
    int ad;  // of the workgroup's, -1: another or none
    bool below;
  };
  auto request = [&](int c) {
    const int s = 64 * c + lane;
    Request r = {0, 0u, -1, false};
    if (s >= a.n_req) return r;
    const Rows R = rows_of(a, s);
    const int ad = adapter_of(a, s);
    r.first = (int)R.r0;
    r.rows = (uint32_t)(R.r1 - R.r0);
    r.below = ad >= 0 && ad < a0;
    if (ad >= a0 && ad < a0 + kOrderAdapters) r.ad = ad - a0;
    return r;
  };
  uint32_t below = 0;  // rows of lower adapters
  for (int c = c0; c < c1; ++c) {
    const Request r = request(c);
    if (r.below) below += r.rows;
    if (r.ad >= 0) atomicAdd(count + r.ad, r.rows);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) below += (uint32_t)__shfl_xor((int)below, d);
  if (lane == 0) sums[wave] = below;
  __syncthreads();
  uint32_t mine[4], total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) total += mine[w] = lds[w * kOrderAdapters + threadIdx.x];
  uint32_t upto = total;  // with the lower lanes'
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t v = (uint32_t)__shfl_up((int)upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) sums[4 + wave] = upto;
  __syncthreads();
  uint32_t start = upto - total;
#pragma unroll
  for (int w = 0; w < 4; ++w) start += sums[w] + (w < wave ? sums[4 + w] : 0u);
  const int ad = a0 + (int)threadIdx.x;
  auto in_n = [&](uint32_t x) { return (int64_t)x < a.n ? (int64_t)x : a.n; };
  if (ad < a.n_ad) to.off[ad] = in_n(start);
  if (ad == a.n_ad - 1) to.off[a.n_ad] = in_n(start + total);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    lds[w * kOrderAdapters + threadIdx.x] = start;
    start += mine[w];
  }
  __syncthreads();
  for (int c = c0; c < c1; ++c) {
    const Request r = request(c);
    const bool in = r.ad >= 0 && r.rows > 0;
    if (!__any(in)) continue;
    uint32_t at = 0;
#pragma unroll 8
    for (int i = 0; i < 64; ++i)  // rows of earlier requests of the 64 with this one's adapter
      if (__builtin_amdgcn_readlane(r.ad, i) == r.ad && i < lane)
        at += (uint32_t)__builtin_amdgcn_readlane((int)r.rows, i);
    if (in) {
      at += count[r.ad];
      atomicAdd(count + r.ad, r.rows);
    }
    constexpr uint32_t kOwn = 16;  // rows that a lane writes by itself
    const bool few = in && r.rows <= kOwn;
    for (uint32_t j = 0; j < kOwn && __any(few && j < r.rows); ++j)
      if (few && j < r.rows && (int64_t)at + j < a.n) to.list[at + j] = r.first + (int)j;
    for (unsigned long long left = __ballot(in && !few); left; left &= left - 1) {
      const int i = __builtin_ctzll(left);
      const int64_t p = (uint32_t)__builtin_amdgcn_readlane((int)at, i);
      const int first = __builtin_amdgcn_readlane(r.first, i);
      int64_t n = (uint32_t)__builtin_amdgcn_readlane((int)r.rows, i);
      if (n > a.n - p) n = a.n - p;
      for (int64_t j = lane; j < n; j += 64) to.list[p + j] = first + (int)j;
    }
  }
}

// ---- transposed weights -----------------------------------------------------------------------

// Up to three batches of matrices in one launch, a 64 x 64 tile per workgroup: whole 16-byte pieces of
// rows in and out where both sizes are multiples of 8, values otherwise.  Bound by memory and its launch: W of
// 4096 x 4096 and an adapter of rank 64, 17.5 us (69 MB, 3.9 TB/s).
__global__ __launch_bounds__(256) void prepare_kernel(AdapterArgs g, TransposeArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[64][72];
  int w = 0;
  uint32_t b = blockIdx.x;
  if (b < a.order_blocks) {
    static_assert(sizeof(tile) >= 4 * kOrderLds, "the counts fit the tile");
    order_rows(g, a.order, reinterpret_cast<uint32_t*>(tile), (int)b * kOrderAdapters);
    return;
  }
  b -= a.order_blocks;
  while (w < 2 && b >= a.job[w].blocks) b -= a.job[w++].blocks;
  const TransposeJob& q = a.job[w];
  const int rows = q.rows, cols = q.cols;
  const uint32_t n_c = (uint32_t)(cols + 63) / 64u, n_r = (uint32_t)(rows + 63) / 64u;
  const int64_t base = (int64_t)(b / (n_c * n_r)) * rows * cols;
  const uint32_t in_m = b % (n_c * n_r);
  const int r0 = (int)(in_m / n_c) * 64, c0 = (int)(in_m % n_c) * 64;
  const uint16_t* in = q.in + base;
  uint16_t* out = q.out + base;
  if (rows % 8 == 0 && cols % 8 == 0) {
    const int x = 8 * (threadIdx.x & 7), y = threadIdx.x >> 3;
#pragma unroll
    for (int i = y; i < 64; i += 32)
      if (r0 + i < rows && c0 + x < cols)
        *reinterpret_cast<u32x4*>(&tile[i][x]) = load16(in + (int64_t)(r0 + i) * cols + c0 + x);
    __syncthreads();
    // thread: 8 rows of one column; a wave's 64 columns of the same rows read LDS without conflicts
    const int c = threadIdx.x & 63;
#pragma unroll
    for (int k = threadIdx.x >> 6; k < 8; k += 4) {
      if (c0 + c >= cols || r0 + 8 * k >= rows) continue;
      u32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = (uint32_t)tile[8 * k + 2 * e][c] | (uint32_t)tile[8 * k + 2 * e + 1][c] << 16;
      *reinterpret_cast<u32x4*>(out + (int64_t)(c0 + c) * rows + r0 + 8 * k) = v;
    }
    return;
  }
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  for (int i = y; i < 64; i += 4)
    if (r0 + i < rows && c0 + x < cols) tile[i][x] = in[(int64_t)(r0 + i) * cols + c0 + x];
  __syncthreads();
  for (int i = y; i < 64; i += 4)
    if (c0 + i < cols && r0 + x < rows) out[(int64_t)(c0 + i) * rows + r0 + x] = tile[x][i];
}

// ---- dA, dB -----------------------------------------------------------------------------------

// Partial sums over up to o.rows rows of one request, or, in calls of many requests, of one adapter by the
// order of order_rows (LIST), so that the parts do not grow with the requests: part[slot][j][c] = sum_t
// L[t,j] M[t,c], 64 ranks and 256 columns per workgroup, 64 columns per wave; rows in tiles of 64 through two
// LDS stages, both operands read by columns.  dA and dB go in one launch.  Bound by x and dy: 13,057 rows of
// 4096 each, rank 64: 45 us (214 MB and 27 MB of parts, 5.4 TB/s).
constexpr int kOuterWaves = 4;

// ranks of a workgroup: in fp16 the other half of the tile's 64 columns is the rest of L (kRest)
template <class T>
constexpr int kOuterRanks = T::kNarrow ? 32 : 64;

template <class T, bool LIST>
__global__ __launch_bounds__(64 * kOuterWaves, 2) void outer_kernel(AdapterArgs a, OuterArgs o) {
  constexpr int kTile = 64 * 128;  // 64 rows of 64 values
  constexpr int kStage = (1 + kOuterWaves) * kTile;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // 2 stages
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rp = (a.r + 15) / 16 * 16;
  const uint32_t n_jb = (uint32_t)(rp + kOuterRanks<T> - 1) / kOuterRanks<T>;
  const int which = blockIdx.x >= o.job[0].blocks;
  const OuterJob& q = o.job[which];
  const uint32_t b0 = blockIdx.x - (which ? o.job[0].blocks : 0u);
  const int cols = q.cols;
  const uint32_t n_cb = (uint32_t)(cols + 64 * kOuterWaves - 1) / (64u * kOuterWaves);
  const int cb = (int)(b0 % n_cb), jb = (int)(b0 / n_cb % n_jb);
  const uint32_t slot = b0 / n_cb / n_jb;
  const int64_t* off = LIST ? o.order.off : a.off;
  const int s = find_seq(off, LIST ? a.n_ad : a.n_req, o.rows, slot);
  const Rows R = rows_of(off, a.n, s);
  const int64_t first =
      R.r0 + ((int64_t)slot - ((uint32_t)R.r0 / (uint32_t)o.rows + (uint32_t)s)) * o.rows;
  const int ad = first >= R.r0 && first < R.r1 ? LIST ? s : adapter_of(a, s) : -1;
  if (cb == 0 && jb == 0 && threadIdx.x == 0) o.slot_adapter[which * o.slots + slot] = ad;
  if (ad < 0) return;
  const int64_t end = R.r1 < first + o.rows ? R.r1 : first + o.rows;

  const int c0 = cb * 64 * kOuterWaves + wave * 64;
  const int j0 = jb * kOuterRanks<T>;
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const TileReads<64> rd(lane);
  const int lr = lane >> 3;  // row of a wave load, 8 rows of 8 chunks
  // With a list, a lane holds the row of the tile that is its own number, read a stage ahead.
  auto rows_at = [&](int64_t t) {
    const uint32_t r = LIST ? (uint32_t)o.order.list[t + lane < end ? t + lane : end - 1] : 0u;
    return (int)(r < (uint32_t)a.n ? r : (uint32_t)a.n - 1u);
  };
  // rows past the end are zero in both tiles; columns past the last repeat it, and their sums are
  // not stored
  auto issue = [&](int buf, int64_t t, int listed) {
    const uint32_t st = LDS_ADDRESS(smem) + buf * kStage;
    const int n = end - t < 64 ? (int)(end - t) : 64;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 8 * j + lr;
      int cc = c0 + 8 * ((lane & 7) ^ swz<64>(r));
      if (cc >= cols) cc = cols - 8;
      const int64_t row = LIST ? (int64_t)__shfl(listed, r) : t + r;
      load_lds16(r < n ? (const void*)(q.m + row * cols + cc) : (const void*)kZero16,
                 st + (1 + wave) * kTile + j * 1024);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = 8 * (2 * wave + j) + lr;
      const int ch = 8 * ((lane & 7) ^ swz<64>(r));
      int cc = j0 + ch % kOuterRanks<T>;
      if (cc >= rp) cc = rp - 8;
      const int64_t row = LIST ? (int64_t)__shfl(listed, r) : t + r;
      load_lds16(r < n ? (const void*)((ch < kOuterRanks<T> ? q.l : q.low) + row * rp + cc) : (const void*)kZero16,
                 st + (2 * wave + j) * 1024);
    }
  };
  issue(0, first, rows_at(first));
  int next = rows_at(first + 64);
  int buf = 0;
#pragma unroll 1
  for (int64_t t = first; t < end; t += 64, buf ^= 1) {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    sync_lds();  // the stage has landed, and nobody reads the other any more
    if (t + 64 < end) {
      issue(buf ^ 1, t + 64, next);
      next = rows_at(t + 128);
    }
    const unsigned char* ls = smem + buf * kStage;
    const unsigned char* ms = ls + (1 + wave) * kTile;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        u32x4 fm[2], fl[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fm[i] = rd.tr_frag(ms, b, st, i);
          fl[i] = rd.tr_frag(ls, b, st, i);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = T::mfma(fm[i], fl[j], acc[i][j]);
      }
  }
  if constexpr (T::kNarrow) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][0][r] += acc[i][1][r] * (1.f / kRest);
  }
#pragma unroll
  for (int j = 0; j < kOuterRanks<T> / 32; ++j) {
    const int jj = j0 + 32 * j + col;
    if (jj >= a.r) continue;
    float* dst = q.part + ((int64_t)slot * rp + jj) * cols;
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

// out[ad] = the sum of its slots' parts, in their order.  A thread per rank and 4 columns; a wave
// looks for the adapter's slots 64 at a time and loads 8 of them together (13 slots of 64 x 4096 twice: 7.8 us,
// 3.5 TB/s).  No atomics: the order of the sum is fixed.
template <class T>
__global__ __launch_bounds__(256) void outer_join_kernel(AdapterArgs a, OuterArgs o) {
  const int which = blockIdx.x >= o.job[0].join_blocks;
  const OuterJob& q = o.job[which];
  const uint32_t b = blockIdx.x - (which ? o.job[0].join_blocks : 0u);
  const int ad = blockIdx.y, cols = q.cols;
  const uint32_t i = b * 256 + threadIdx.x;
  const uint32_t per = (uint32_t)cols / 4u;
  const int j = (int)(i / per), c = 4 * (int)(i % per);
  const bool live = j < a.r;
  const int rp = (a.r + 15) / 16 * 16, lane = threadIdx.x & 63;
  const float* src = q.part + (int64_t)(live ? j : 0) * cols + c;
  const int32_t* slots = o.slot_adapter + which * o.slots;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t base = 0; base < o.slots; base += 64) {
    unsigned long long mine = __ballot(base + lane < o.slots && slots[base + lane] == ad);
    while (mine) {
      f32x4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (mine) {
          const uint32_t s = base + __builtin_ctzll(mine);
          v[k] = *reinterpret_cast<const f32x4*>(src + (int64_t)s * rp * cols);
          mine &= mine - 1;
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += v[k];
    }
  }
  if (!live) return;
  uint16_t* out = q.out;
  if (q.transposed) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      out[((int64_t)ad * cols + c + e) * a.r + j] = (uint16_t)T::pack(sum[e], 0.f);
  } else {
    *reinterpret_cast<uint2*>(out + ((int64_t)ad * a.r + j) * cols + c) =
        uint2{T::pack(sum[0], sum[1]), T::pack(sum[2], sum[3])};
  }
}

// The dynamic LDS of a kernel beyond the default limit.
hipError_t allow_lds(const void* fn, int lds) {
  return lds > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds) : hipSuccess;
}

template <class T, int NB, int XB, int W>
hipError_t shrink_as(const ShrinkArgs& p, int count, hipStream_t s) {
  const AdapterArgs& a = p.job[0].a;
  constexpr int lds = W * WaveProduct<T, NB, XB>::kBytes;
  const hipError_t e = allow_lds((const void*)shrink_kernel<T, NB, XB, W>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((shrink_kernel<T, NB, XB, W>),
                     dim3((unsigned)(a.n / (32 * XB) + a.n_req), (unsigned)(a.r + 32 * NB - 1) / (32 * NB),
                          (unsigned)count),
                     dim3(64 * W), lds, s, p);
  return hipGetLastError();
}

// By the number of tiles of 32 rows (k 4096, us of a call with a small W):
//   8 waves on 32 ranks each while all of these workgroups run at a time: rank 128, 32 rows 19 (2 waves on
//     all the ranks: 37), 2,048 rows 38 (50); rank 64, 32 rows 17 (6 waves on 64 ranks: 18), 1,024 rows
//     27 (30), 4,096 rows 40 (36); rank 16, 8,192 rows 42 (4 waves: 45), 10,000 rows 66 (64)
//   then as many waves as two workgroups per CU allow on all the ranks.  Ranks above 32 read as much of A
//     as of x per 32 rows and more: there 64 rows share it, where they fill the chip: 10,000 rows of
//     rank 64 68 (75).
template <class T>
hipError_t shrink(const ShrinkArgs& p, int count, hipStream_t s) {
  const AdapterArgs& a = p.job[0].a;
  const int64_t tiles = a.n / 32 + a.n_req;
  if (tiles * ((a.r + 31) / 32) <= (a.r <= 64 ? 256 : 512)) return shrink_as<T, 1, 1, 8>(p, count, s);
  if (a.r <= 32) return shrink_as<T, 1, 1, 4>(p, count, s);
  if (a.r <= 64)
    return tiles <= 256 ? shrink_as<T, 2, 1, 6>(p, count, s) : shrink_as<T, 2, 2, 4>(p, count, s);
  return shrink_as<T, 4, 1, 2>(p, count, s);
}

template <class T, int BT, int BM, int WT, int WM, int NST, int MINB>
hipError_t expand_as(const AdapterArgs& a, const uint16_t* h, uint16_t* y, hipStream_t s) {
  const int n_m = (a.m + BM - 1) / BM;
  const int64_t grid = (a.n - a.row0 + BT - 1) / BT * n_m;
  constexpr int lds = NST * (BT + BM) * 128;
  const hipError_t e = allow_lds((const void*)expand_kernel<T, BT, BM, WT, WM, NST, MINB>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((expand_kernel<T, BT, BM, WT, WM, NST, MINB>), dim3((unsigned)grid),
                     dim3(64 * WT * WM), lds, s, a, h, y, n_m);
  return hipGetLastError();
}

template <class T, int BM>
hipError_t few_as(const AdapterArgs& a, const uint16_t* h, uint16_t* y, hipStream_t s) {
  const int n_m = (a.m + BM - 1) / BM;
  constexpr int lds = kFewLds<T, BM>;
  const hipError_t e = allow_lds((const void*)expand_few_kernel<T, BM>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((expand_few_kernel<T, BM>), dim3((unsigned)((a.n + 31) / 32 * n_m)),
                     dim3(kFewThreads<BM>), lds, s, a, h, y, n_m);
  return hipGetLastError();
}

// The tile of y, by the number of tiles that the call has (the projections alone, us):
//   32 x 16    up to 128 tiles of 32 x 32, which leave CUs idle: 4096 -> 4096, 1 row 14.9 (32 x 32: 15.5), 32
//              rows 16.9 (19.1), 64 rows (256 tiles) 25 (19); 14336 -> 4096, 32 rows 39 (43)
//   32 x 32    up to 384 of them: 4096 -> 4096, 64 rows (256 tiles) 19 (64 x 64: 31), 96 rows (384) 29 (32),
//              256 rows (2,048) 49 (30); 4096 -> 16384, 8 rows (512) 38 (34), 33 rows (1,024) 67 (35)
//   64 x 64    otherwise, until
//   128 x 128  there are 160 of these: 4096 -> 4096, 512 rows (128 tiles) 39 (64 x 64: 36), 768 rows (192)
//              42 (55), 1,024 rows (256) 47 (62)
//   256 x 256  there are 144 of these: 4096 -> 4096, 2,048 rows (128 tiles) 87 (128 x 128: 83), 2,560 rows
//              (160) 93 (111), 4,096 rows (256) 121 (157)
// and a last round (of 256, one a CU) of up to 112 of the largest is left to the next size: 512 tiles and 64
// more 274 (305 without that), 96 more 303 (307), 128 more 312 (308), 160 more 341 (315).
constexpr int kHalfTo = 128, kFewTo = 384, kMidFrom = 160, kWideFrom = 144, kLastRound = 112;

template <class T>
hipError_t expand(AdapterArgs a, const uint16_t* h, uint16_t* y, hipStream_t s) {
  auto tiles = [&](int b) { return (a.n - a.row0 + b - 1) / b * ((a.m + b - 1) / b); };
  if (tiles(32) <= kFewTo) return tiles(32) <= kHalfTo ? few_as<T, 16>(a, h, y, s) : few_as<T, 32>(a, h, y, s);
  if (tiles(256) >= kWideFrom) {
    const int64_t n_m = (a.m + 255) / 256, rest = tiles(256) % 256;
    const int64_t rows = (tiles(256) - rest) / n_m * 256;  // of the whole rounds
    AdapterArgs w = a;
    if (rest > 0 && rest <= kLastRound && rows > 0) w.n = rows;
    const hipError_t e = expand_as<T, 256, 256, 4, 2, 2, 1>(w, h, y, s);
    if (e != hipSuccess || w.n == a.n) return e;
    a.row0 = rows;
  }
  if (tiles(128) >= kMidFrom || a.row0 > 0) return expand_as<T, 128, 128, 4, 2, 4, 1>(a, h, y, s);
  return expand_as<T, 64, 64, 2, 2, 4, 2>(a, h, y, s);
}

template <class T>
hipError_t outer(const AdapterArgs& a, OuterArgs o, hipStream_t s) {
  const int rp = adapter_rank_pad(a.r), n_jb = (rp + kOuterRanks<T> - 1) / kOuterRanks<T>;
  o.rows = adapter_outer_rows(a.n, a.k, a.m);
  o.slots = (uint32_t)adapter_outer_slots(a.n, a.n_req, a.n_ad, a.k, a.m, a.r);
  uint32_t blocks = 0, join_blocks = 0;
  for (OuterJob& q : o.job) {
    q.blocks = q.join_blocks = 0;
    if (!q.out) continue;
    q.blocks = o.slots * (uint32_t)((q.cols + 64 * kOuterWaves - 1) / (64 * kOuterWaves)) * n_jb;
    q.join_blocks = (uint32_t)(((int64_t)a.r * (q.cols / 4) + 255) / 256);
    blocks += q.blocks;
    join_blocks += q.join_blocks;
  }
  if (join_blocks == 0) return hipSuccess;
  hipError_t e = hipSuccess;
  if (blocks > 0) {
    constexpr int lds = 2 * (1 + kOuterWaves) * 64 * 128;
    auto run = [&](auto kernel) {
      const hipError_t f = allow_lds((const void*)kernel, lds);
      if (f != hipSuccess) return f;
      hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * kOuterWaves), lds, s, a, o);
      return hipGetLastError();
    };
    e = adapter_ordered(a.n, a.n_req, a.n_ad, a.k, a.m, a.r) ? run(outer_kernel<T, true>) : run(outer_kernel<T, false>);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((outer_join_kernel<T>), dim3(join_blocks, (unsigned)a.n_ad), dim3(256), 0, s, a, o);
  return hipGetLastError();
}

}  // namespace

// 1,024 rows a slot where that leaves most of a round of workgroups (two per CU), 512 otherwise: more
// rows, fewer partial sums to write and join.  All of the gradients, rank 16, 1,024 (512) rows a slot:
// 4096 -> 4096, 13,057 rows (384 workgroups) 444 us (452), 8,192 rows (256) 288 (287); 1024 -> 1024, 40,000
// rows (312) 151 (156), 13,057 rows (96) 67 (63).
int adapter_outer_rows(int64_t n, int k, int m) { return (n / 1024) * ((k + m) / 256) >= 300 ? 1024 : 512; }

// Slots of one request each where that is not many: the order takes 9 us (the prepare kernel's and the wait
// for the list in the outer kernel's), which the parts of the slots that it saves outweigh from 12 MB on.  All of
// the gradients and the forward, us ordered (by request): 768 -> 768, rank 8, 4 adapters, 64 requests (6 MB) 48
// (47), 256 (25 MB) 56 (66), 1,024 of 2 rows 86 (130); 768 -> 2304, 37 requests of 5 (6 MB) 60 (51); 4096 -> 4096,
// rank 16, 32 requests of 4 adapters (15 MB) 88 (94), 64 of 16 in 13,063 rows (25 MB) 919 (918), 4,096 of one row,
// 8 adapters (2.1 GB) 596 (1,980).
constexpr int64_t kOrderFrom = 12 << 20;  // bytes

bool adapter_ordered(int64_t n, int n_req, int n_ad, int k, int m, int r) {
  if (n == 0 || n_ad == 0 || n_req <= n_ad) return false;
  return (int64_t)(n_req - n_ad) * adapter_rank_pad(r) * (k + m) * (int64_t)sizeof(float) >= kOrderFrom;
}

int64_t adapter_outer_slots(int64_t n, int n_req, int n_ad, int k, int m, int r) {
  if (n == 0 || n_req == 0 || n_ad == 0) return 0;
  return n / adapter_outer_rows(n, k, m) + (adapter_ordered(n, n_req, n_ad, k, m, r) ? n_ad : n_req);
}

// (The tiles of y are 256 x 256 by 512 threads in every call of this size, those of h 32 rows by 256.)
bool adapters_fit(int64_t n, int k, int m, int r, int n_ad, int n_req, bool grads) {
  auto blocks = [](int64_t size, int of) { return (size + of - 1) / of; };
  const int64_t wide = k > m ? k : m;
  if (!launch_fits(blocks(n, 256) * blocks(grads ? wide : m, 256), 512)) return false;
  if (!launch_fits(blocks(n, 32) + n_req, 256)) return false;
  if (!grads) return true;
  const int64_t prepare =
      blocks(n_ad, kOrderAdapters) + blocks(m, 64) * blocks(k, 64) + n_ad * blocks(r, 64) * (blocks(k, 64) + blocks(m, 64));
  const int64_t outer = adapter_outer_slots(n, n_req, n_ad, k, m, r) * blocks(adapter_rank_pad(r), 32) *
                        (blocks(k, 64 * kOuterWaves) + blocks(m, 64 * kOuterWaves));
  return launch_fits(prepare, 256) && launch_fits(outer, 64 * kOuterWaves);
}

hipError_t launch_adapter_shrink(const ShrinkJob* jobs, int count, hipStream_t stream) {
  const AdapterArgs& a = jobs[0].a;
  if (a.n == 0 || a.n_req == 0) return hipSuccess;
  const ShrinkArgs p = {{jobs[0], jobs[count - 1]}};
  return a.f16 ? shrink<HalfF16>(p, count, stream) : shrink<HalfBf16>(p, count, stream);
}

hipError_t launch_adapter_expand(const AdapterArgs& a, const uint16_t* h, uint16_t* y,
                                 hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  return a.f16 ? expand<HalfF16>(a, h, y, stream) : expand<HalfBf16>(a, h, y, stream);
}

hipError_t launch_adapter_prepare(const AdapterArgs& g, TransposeArgs a, hipStream_t stream) {
  a.order_blocks = a.order.list ? (uint32_t)((g.n_ad + kOrderAdapters - 1) / kOrderAdapters) : 0u;
  int64_t blocks = a.order_blocks;
  for (TransposeJob& q : a.job) {
    q.blocks = (uint32_t)(q.count * ((q.rows + 63) / 64) * ((q.cols + 63) / 64));
    blocks += q.blocks;
  }
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(prepare_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, g, a);
  return hipGetLastError();
}

hipError_t launch_adapter_outer(const AdapterArgs& a, const OuterArgs& o, hipStream_t stream) {
  if (a.n_ad == 0) return hipSuccess;
  return a.f16 ? outer<HalfF16>(a, o, stream) : outer<HalfBf16>(a, o, stream);
}

}  // namespace hpr
