// Products of rows with rows, out[t][m] = <x_t, w_m>, of 16-bit operands on the matrix cores: a workgroup's
// tile, and a wave's own part.  Shared by the encoder's projections.
//
// W's rows are the rows of the matrix product, so that a lane holds values of one row of x: entry e of block
// (i, j) is row 8 (e / 4) + 4 half + e % 4 of W's block i and row lane & 31 of x's block j.
#pragma once

#include <type_traits>

#include "common.h"
#include "half.h"
#include "tiles.h"

namespace hpr {

__device__ __attribute__((aligned(16))) const uint32_t kZero16[4] = {0u, 0u, 0u, 0u};

// Rows of the right operand.  A paired tile (PAIR) takes its rows from two matrices, the same rows of each:
// one half of every wave's rows from w[0], the other from w[1].
struct PanelW {
  const uint16_t* w[2];  // first rows (w[1] of a paired tile alone)
  int ld;                // elements from a row to the next
  int last;              // last valid row, which the rows past it repeat
};

// A right operand by columns: value c of k is row c of w[0] below `half`, row c - half of w[1] from there; the tile's
// columns begin at those rows' own.
struct PanelT {
  const uint16_t* w[2];
  int ld;           // elements from a row to the next
  int last;         // last valid column, whose chunk of 8 the chunks past it repeat
  int first, half;  // k begins at value `first`
  __device__ __forceinline__ const uint16_t* row(int c) const {
    return c < half ? w[0] + (int64_t)c * ld : w[1] + (int64_t)(c - half) * ld;
  }
};

// ---- a wave's own product ----------------------------------------------------------------------

// acc[b][c] = rows [32 b, 32 b + 32) of P times rows [32 c, + 32) of X, over stages [kk0, kk1) of 64 values,
// by one wave: its NST LDS stages are its own, so waves that split k run without a barrier.  Whole 128-byte
// lines go straight to LDS (operands read from memory by lanes touch twice as many lines a load: a token's
// projection took 22 us that way).  Of P, ROWS rows are loaded; the results of the rest of its last 32 are
// not to be used (their operands are what LDS holds past the stage, of this wave's or another's).  STREAM: P is read
// once by the whole call, and keeps out of the caches.
template <class T, int NB, int XB, int NST = 2, int ROWS = 32 * NB, bool PAIR = false, bool STREAM = false>
struct WaveProduct {
  static constexpr int kStage = XB * 4096 + ROWS * 128;
  static constexpr int kBytes = NST * kStage;
  static constexpr int kPast = (32 * NB - ROWS) * 128;  // LDS read past the stages
  static constexpr int kX = 4 * XB, kLoads = 4 * XB + ROWS / 8;
  // x: first row; x_last: its last valid row, which the rows past it repeat
  static __device__ __forceinline__ void run(const uint16_t* x, int x_ld, int x_last, const PanelW& p,
                                             int k, int kk0, int kk1, unsigned char* lds, int lane,
                                             f32x16 (&acc)[NB][XB]) {
    static_assert(!PAIR || ROWS % 16 == 0, "a load's eight rows are of one matrix");
    const __amdgpu_buffer_rsrc_t rx = tile_rsrc(x), rp = tile_rsrc(p.w[0]), rq = tile_rsrc(p.w[PAIR]);
    const TileReads<64> rd(lane);
    int off[kLoads], chunk[kLoads];
    auto second = [](int j) { return PAIR && j >= kX + ROWS / 16; };  // a load of w[1]
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      int r = 8 * (j < kX ? j : j - kX) + (lane >> 3);
      chunk[j] = ((lane & 7) ^ swz<64>(r)) * 8;
      if (second(j)) r -= ROWS / 2;
      const int last = j < kX ? x_last : p.last;
      off[j] = (r < last ? r : last) * (j < kX ? x_ld : p.ld) * 2 + chunk[j] * 2;
    }
    const int whole = k / 64;
    auto issue = [&](int buf, int kk) {
      unsigned char* st = lds + buf * kStage;
      if (kk < whole) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          if (j < kX)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void_t*)(st + j * 1024), 16, off[j], kk * 128, 0, 0);
          else  // (2: nt)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second(j) ? rq : rp, (lds_void_t*)(st + j * 1024), 16, off[j],
                                                     kk * 128, 0, STREAM ? 2 : 0);
        }
      } else {  // the end of k: chunks past it read zeros
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const char* src = (const char*)(j < kX ? x : p.w[second(j)]) + off[j] + kk * 128;
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

// ---- a workgroup's product ---------------------------------------------------------------------

// Tile of BT rows of x by BM rows of W, WT x WM waves, k in stages of 64 through NST LDS stages.  Wave
// (wt, wm) holds the rows [32 kTb wt, + 32 kTb) of x and [32 kMb wm, + 32 kMb) of W.
template <class T, int BT, int BM, int WT, int WM, int NST>
struct TileProduct {
  static constexpr int kW = WT * WM;
  static constexpr int kTb = BT / 32 / WT, kMb = BM / 32 / WM;  // blocks per wave
  static constexpr int kXBytes = BT * 128, kWBytes = BM * 128, kStage = kXBytes + kWBytes;
  static constexpr int kLds = NST * kStage;
  typedef f32x16 Acc[kMb][kTb];

  // x: first row of the tile.  `first` is called between the first stages' loads and the products, to add
  // to acc (zero there).  LDS is free for the caller when this returns.
  template <class First>
  static __device__ __forceinline__ void run(const uint16_t* xb, int ldx, int last_t, const PanelW& w, int k,
                                             unsigned char* smem, int wave, int lane, Acc& acc,
                                             First&& first) {
    const int wt = wave % WT, wm = wave / WT;
    const TileReads<64> rd(lane);
    const TileLoad<64, BT, kW> lx(wave, lane, 8);
    const TileLoad<64, BM, kW> lw(wave, lane, 8);
    constexpr int kLoads = lx.kLoads + lw.kLoads;
    const __amdgpu_buffer_rsrc_t rx = tile_rsrc(xb), rw = tile_rsrc(w.w[0]);
    int ox[lx.kLoads], ow[lw.kLoads];
#pragma unroll
    for (int j = 0; j < lx.kLoads; ++j)
      ox[j] = (lx.row[j] < last_t ? lx.row[j] : last_t) * ldx * 2 + lx.chunk[j];
#pragma unroll
    for (int j = 0; j < lw.kLoads; ++j)
      ow[j] = (lw.row[j] < w.last ? lw.row[j] : w.last) * w.ld * 2 + lw.chunk[j];
    const int nk = (k + 63) / 64, nk_full = k / 64;
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
          const bool in = kk * 64 + lx.chunk[j] / 2 < k;
          const void* p = in ? (const void*)((const char*)xb + ox[j] + kk * 128) : (const void*)kZero16;
          __builtin_amdgcn_global_load_lds((glb_void_t*)p, (lds_void_t*)(st + (wave * lx.kLoads + j) * 1024),
                                           16, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < lw.kLoads; ++j) {
          const bool in = kk * 64 + lw.chunk[j] / 2 < k;
          const char* wb = (const char*)w.w[0];
          const void* p = in ? (const void*)(wb + ow[j] + kk * 128) : (const void*)kZero16;
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

#pragma unroll
    for (int i = 0; i < kMb; ++i)
#pragma unroll
      for (int j = 0; j < kTb; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    first(acc);

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
    // no load may still target LDS when it is reused or ends, and nobody may still read it
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    sync_lds();
  }
};

// Tile of block b of a grid of n_t row tiles by n_m column tiles.  An XCD walks a contiguous run of tiles,
// four row tiles abreast: the tiles that it holds at a time (32 of the widest) read 4 row tiles and 8 column
// tiles, not 1 or 2 and all the columns.
struct TileAt {
  uint32_t t;
  int m;
};
__device__ __forceinline__ TileAt tile_of(uint32_t lin, uint32_t n_t, int n_m) {
  const uint32_t g0 = lin / (4u * n_m) * 4u, in_g = lin - g0 * n_m;
  const uint32_t abreast = n_t - g0 < 4u ? n_t - g0 : 4u;
  return {g0 + in_g % abreast, (int)(in_g / abreast)};
}
__device__ __forceinline__ TileAt tile_at(uint32_t block, uint32_t blocks, uint32_t n_t, int n_m) {
  return tile_of((uint32_t)xcd_linear(block, blocks), n_t, n_m);
}

// ---- a workgroup's product, in blocks of 16 ------------------------------------------------------

// The same in 16x16x32 products.  On operands that are not zero the card's power limit holds the clock, and these
// take less of it than 32x32x16: from registers alone, bf16 normal values, 1.97 PFLOP/s against 1.68 (zeros: 2.44
// and 2.40).  Wave (wt, wm) holds the rows [16 kT wt, + 16 kT) of x and [16 kM wm, + 16 kM) of W; entry e of block
// (i, j) is row 4 (lane / 16) + e of W's block i and row lane % 16 of x's block j.  Of a paired tile (PAIR) the
// blocks i < kM / 2 are columns of w[0], the others the same columns of w[1].
//
// k goes in stages of 64 values (whole 128-byte lines: half lines ask the L2 for twice as many) through LDS, x's
// through a ring of NX, W's through one of NW <= NX.  A stage is two k-steps, whose operands a wave holds in
// registers: while it multiplies one, it reads the other, and loads what takes the place of the stage before.  One
// barrier a stage, between its k-steps: from there on nobody reads the stage's LDS.  Reads and loads stand between
// the products one at a time, because a run of them holds the matrix cores up.
//
// An XCD's tiles (tile_at) go through k together, so that every stage is new to its L2, and its loads would wait for
// memory.  In the largest tile one more load a wave touches lines kTouch stages ahead: the four row tiles share the
// columns' panel, and each touches a quarter of its rows' lines, as the eight column tiles do an eighth of the
// rows'.  (Zeros as operands 1,990 -> 1,745 us, 13,063 rows, 4096 -> 14336; the gradients of 6,529 rows 4,010 ->
// 3,890; on random operands the forward is at the power limit without it.)
//
// W by columns (PanelT): a stage is 64 rows of BM values, and the matrix cores' operands, eight rows of a column a
// lane, are read with two transposing reads.  Such a read takes 32 bytes of eight rows a cycle (four, and the four
// that are eight or so further): their chunks are placed (by_rows) so that these are all of the banks.  Its loads are
// written out (load_lds16): before a transposing read the compiler waits for every load to LDS that it knows of (x's
// gradients of 6,529 rows, 4096 -> 14336 3,450 us, without the waits 2,393).  It touches no lines ahead: the touched
// value's wait would be for all of those loads too.
template <class T, int BT, int BM, int WT, int WM, int NX, int NW, bool PAIR = false>
struct TileProduct16 {
  static constexpr int kW = WT * WM;
  static constexpr int kT = BT / 16 / WT, kM = BM / 16 / WM;  // blocks per wave
  static constexpr int kX = BT * 128, kStageW = BM * 128;     // bytes of a stage of each
  static constexpr int kLds = NX * kX + NW * kStageW;
  static constexpr int kLx = BT / 8 / kW, kLw = BM / 8 / kW;  // loads of a wave for a stage
  static constexpr int kCols = PAIR ? BM / 2 : BM;            // columns of the output
  static constexpr int kWaveCols = kCols / WM;
  static constexpr int kThreads = 64 * kW, kRows = BT, kWt = WT;
  static __device__ __forceinline__ int in_stage(int load, int lane) {  // row of a lane's chunk, by columns
    return load * (512 / BM) + lane / (BM / 8);
  }
  static constexpr int kTouch = BT == 256 && BM == 256 && kW == 8 ? 4 : 0;  // (0: none)
  static_assert(!PAIR || kM % 2 == 0, "a wave holds both halves of its columns");
  static_assert(NW >= 2 && (NX == NW || NX == NW + 1) && kLds <= 160 * 1024, "the waits below");
  typedef f32x4 Acc[kM][kT];
  struct Frags {
    u32x4 x[kT], w[kM];
  };

  // Chunk c of row r of a stage by columns is stored at position c ^ by_rows(r) of its row.
  static __device__ __forceinline__ int by_rows(int r) { return ((r & 3) | (((r >> 3) ^ (r >> 4)) & 1) << 2) << 1; }

  // x: first row of the tile, of k values.  nk: stages, at least k / 64 (groups of waves that split k call this
  // with the same number, because of its barriers).  LDS is free for the caller when this returns.
  template <class Panel>
  static __device__ __forceinline__ void run(const uint16_t* xb, int ldx, int last_t, const Panel& w, int k, int nk,
                                             TileAt tile, unsigned char* smem, int wave, int lane, Acc& acc) {
    constexpr bool kByCols = std::is_same<Panel, PanelT>::value;
    static_assert(!kByCols || (!PAIR && BM >= 128), "by_rows needs 16 chunks a row");
    constexpr int kTouches = kByCols ? 0 : kTouch;
    const int wt = wave % WT, wm = wave / WT;
    const TileLoad<64, BT, kW, true> lx(wave, lane, 8);
    const TileLoad<64, BM, kW, true> lw(wave, lane, 8);
    const __amdgpu_buffer_rsrc_t rx = tile_rsrc(xb), rw0 = tile_rsrc(w.w[0]), rw1 = tile_rsrc(w.w[PAIR]);
    // the eight rows of a wave load are of one half of a wave's rows
    auto second = [&](int j) { return PAIR && (wave * kLw + j) * 8 % (BM / WM) >= kWaveCols; };
    int ox[kLx], ow[kLw];
#pragma unroll
    for (int j = 0; j < kLx; ++j) ox[j] = (lx.row[j] < last_t ? lx.row[j] : last_t) * ldx * 2 + lx.chunk[j];
#pragma unroll
    for (int j = 0; j < kLw; ++j) {
      if constexpr (kByCols) {
        constexpr int kCh = BM / 8;
        const int r = in_stage(wave * kLw + j, lane), c = (lane % kCh) ^ by_rows(r), last = w.last / 8;
        ow[j] = r * w.ld * 2 + (c < last ? c : last) * 16;
        continue;
      }
      const int row = PAIR ? lw.row[j] / (BM / WM) * kWaveCols + lw.row[j] % kWaveCols : lw.row[j];
      ow[j] = (row < w.last ? row : w.last) * w.ld * 2 + lw.chunk[j];
    }
    // the stages before the first that leaves k or (by columns) has rows of both matrices
    int nk_full = k / 64;
    if constexpr (kByCols) {
      const int left = w.half - w.first;
      if (left > 0 && left % 64 != 0 && left / 64 < nk_full) nk_full = left / 64;
    }
    unsigned char* const ring_w = smem + NX * kX;
    // Load j of x's or W's stage kk into slot `slot` of its ring.  Chunks past the end of k read zeros, so past the
    // last stage too (the rings keep their numbers of loads in flight); WHOLE: the stage is one of nk_full.
    auto load = [&](auto whole, auto of_x, int slot, int kk, int j) __attribute__((always_inline)) {
      unsigned char* to;
      if constexpr (of_x()) to = smem + slot * kX + (wave * kLx + j) * 1024;
      else to = ring_w + slot * kStageW + (wave * kLw + j) * 1024;
      if constexpr (kByCols && whole()) {
        const uint32_t at = (uint32_t)(uintptr_t)(lds_void_t*)to;
        if constexpr (of_x()) load_lds16(rsrc_of(xb), at, (uint32_t)(ox[j] + kk * 128));
        else if constexpr (kByCols) load_lds16(rsrc_of(w.row(w.first + kk * 64)), at, (uint32_t)ow[j]);
      } else if constexpr (whole()) {
        if constexpr (of_x())
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void_t*)to, 16, ox[j], kk * 128, 0, 0);
        else
          __builtin_amdgcn_raw_ptr_buffer_load_lds(second(j) ? rw1 : rw0, (lds_void_t*)to, 16, ow[j], kk * 128, 0, 0);
      } else {
        const void* p = nullptr;
        if constexpr (of_x()) {
          p = kk * 64 + lx.chunk[j] / 2 < k ? (const void*)((const char*)xb + ox[j] + kk * 128) : (const void*)kZero16;
        } else if constexpr (kByCols) {
          const int r = in_stage(wave * kLw + j, lane), c = kk * 64 + r;
          p = c < k ? (const void*)((const char*)w.row(w.first + c) + (ow[j] - r * w.ld * 2)) : (const void*)kZero16;
        } else {
          p = kk * 64 + lw.chunk[j] / 2 < k ? (const void*)((const char*)w.w[second(j)] + ow[j] + kk * 128)
                                            : (const void*)kZero16;
        }
        if constexpr (kByCols) load_lds16(p, (uint32_t)(uintptr_t)(lds_void_t*)to);
        else __builtin_amdgcn_global_load_lds((glb_void_t*)p, (lds_void_t*)to, 16, 0, 0);
      }
    };
    auto load_all = [&](auto of_x, int slot, int kk) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < (of_x() ? kLx : kLw); ++j) {
        if (kk < nk_full) load(std::true_type(), of_x, slot, kk, j);
        else load(std::false_type(), of_x, slot, kk, j);
      }
    };
#pragma unroll
    for (int s = 0; s < NW; ++s) {
      load_all(std::false_type(), s, s);
      if (s < NX - 1) load_all(std::true_type(), s, s);
    }
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
      for (int j = 0; j < kT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // lines to touch: of eight rows of W in the first lanes, of four of x in the next, and those again
    const char* touch = nullptr;
    uint32_t touched = 0;
    if constexpr (kTouches > 0) {
      auto row_of = [](int row, int last) { return row < last ? row : last; };
      const int of_w = (int)(tile.t & 3u) * 64 + wave * 8 + (lane & 7);
      const int of_x = row_of((tile.m & 7) * 32 + wave * 4 + (lane & 3), last_t);
      const bool up = PAIR && of_w % (BM / WM) >= kWaveCols;
      const int in_w = row_of(PAIR ? of_w / (BM / WM) * kWaveCols + of_w % kWaveCols : of_w, w.last);
      touch = lane < 8 ? (const char*)w.w[up] + (int64_t)in_w * w.ld * 2 : (const char*)xb + (int64_t)of_x * ldx * 2;
    }
    // chunk 4 s + lane / 16 of row lane % 16 of a block of 16 rows, of k-step s
    const int r = lane & 15, at0 = r * 128 + (((lane >> 4) ^ swz16(r)) << 4);
    const unsigned char* const own_x = smem + wt * kT * 2048;
    const unsigned char* const own_w = kByCols ? ring_w : ring_w + wm * kM * 2048;
    // by columns: of block b the rows 8 (lane / 16) + lane % 16 / 4, and four further, of k-step s
    const int rt = 8 * (lane >> 4) + ((lane & 15) >> 2);
    const int at_t = rt * BM * 2 + ((((2 * wm * kM) ^ by_rows(rt)) | ((lane & 3) >> 1)) << 4) + ((lane & 1) << 3);
    auto read = [&](int slot_x, int slot_w, int s, Frags& f, int b) __attribute__((always_inline)) {
      const int at = at0 ^ (s << 6);
      if (b < kT) f.x[b] = *reinterpret_cast<const u32x4*>(own_x + slot_x * kX + at + b * 2048);
      else if constexpr (kByCols) {
        typedef short v4s __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4s lds_v4s;
        typedef uint32_t v2u __attribute__((ext_vector_type(2)));
        const unsigned char* p = own_w + slot_w * kStageW + (at_t ^ ((b - kT) << 5)) + s * 64 * BM;
        const v2u lo = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p));
        const v2u hi = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 8 * BM)));
        f.w[b - kT] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      } else f.w[b - kT] = *reinterpret_cast<const u32x4*>(own_w + slot_w * kStageW + at + (b - kT) * 2048);
    };
    constexpr int kReads = kT + kM, kProducts = kT * kM;
    // The products of `now`; between them the reads of k-step s of (slot_x, slot_w), and loads of a stage kk.
    auto step = [&](auto whole, auto of_x, int slot, int kk, int slot_x, int slot_w, int s, const Frags& now,
                    Frags& then) __attribute__((always_inline)) {
      constexpr int kLoads = of_x() ? kLx : kLw;
#pragma unroll
      for (int p = 0; p < kProducts; ++p) {
        const int i = p / kT, j = i & 1 ? kT - 1 - p % kT : p % kT;
        acc[i][j] = T::mfma16(now.w[i], now.x[j], acc[i][j]);
        // (loops of constant length, which the compiler unrolls)
#pragma unroll
        for (int q = 0; q < kReads; ++q)
          if (p == q * kProducts / kReads) read(slot_x, slot_w, s, then, q);
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
          if (p == l * kProducts / kLoads) load(whole, of_x, slot, kk, l);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // Loads that may be on their way when a stage's have landed: at first, and (of x's and W's last, the older
    // one's) at a barrier, before which stage kk - 1 + NX of x and kk - 1 + NW of W are the last that were begun.
    constexpr int kFirst = (NW - 1) * kLw + (NX - 2) * kLx;
    constexpr int kBehind = NX == NW ? (NX - 2) * (kLx + kLw) : (NW - 1) * kLx + (NW - 2) * kLw;
    Frags f0, f1;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(kFirst));
    sync_lds();
#pragma unroll
    for (int q = 0; q < kReads; ++q) read(0, 0, 0, f0, q);
    const int whole = nk_full < nk ? nk_full : nk;
    int kk = 0, sx = 0, sw = 0, before = NX - 1;  // the stage's slots, and that of x's stage before
    auto turn = [&](auto whole) __attribute__((always_inline)) {
      step(whole, std::true_type(), before, kk - 1 + NX, sx, sw, 1, f0, f1);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(kBehind));
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      sync_lds();  // the next stage has landed, and nobody reads this one any more
      if constexpr (kTouches > 0) {
        // (the one before has arrived: it is older than what the wait above was for)
        asm volatile("" : : "v"(touched));
        if constexpr (whole()) {
          const int stage = kk + kTouch < nk_full ? kk + kTouch : nk_full - 1;
          touched = *reinterpret_cast<const uint32_t*>(touch + stage * 128);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      const int slot = sw;
      before = sx;
      sx = sx + 1 < NX ? sx + 1 : 0;
      sw = sw + 1 < NW ? sw + 1 : 0;
      step(whole, std::false_type(), slot, kk + NW, sx, sw, 0, f1, f0);
    };
#pragma unroll 1
    for (; kk + NX < whole; ++kk) turn(std::true_type());
#pragma unroll 1
    for (; kk < nk; ++kk) turn(std::false_type());
    if constexpr (kTouches > 0) asm volatile("" : : "v"(touched));
    // no load may still target LDS when it is reused or ends, and nobody may still read it
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    sync_lds();
  }
};

// The product of a tile by G groups of waves, each of which has its own rings and a G-th of k's stages.  In the end
// the sums of all are group 0's (in the groups' order), whose waves go on (true); the others are done.
template <class P, int G>
__device__ __forceinline__ bool grouped(const uint16_t* xb, int ldx, int last_t, const PanelW& w, int k, TileAt tile,
                                        unsigned char* smem, int wave, int lane, typename P::Acc& acc) {
  const int stages = (k + 63) / 64, each = (stages + G - 1) / G;
  const int group = wave / P::kW, in = wave % P::kW, first = group * each * 64;
  const int left = k - first < each * 64 ? k - first : each * 64;
  P::run(xb + first, ldx, last_t, PanelW{{w.w[0] + first, w.w[1] + first}, w.ld, w.last}, G > 1 ? (left > 0 ? left : 0) : k,
         each, tile, smem + group * P::kLds, in, lane, acc);
  if constexpr (G > 1) {
    constexpr int kOwn = P::kM * P::kT * 1024;  // bytes of a wave's sums
    static_assert((G - 1) * P::kW * kOwn <= G * P::kLds, "the sums fit the rings");
    f32x4* mine = reinterpret_cast<f32x4*>(smem + ((group - 1) * P::kW + in) * kOwn);
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < P::kM; ++i)
#pragma unroll
        for (int j = 0; j < P::kT; ++j) mine[(i * P::kT + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (group > 0) return false;
#pragma unroll
    for (int g = 1; g < G; ++g) {
      const f32x4* from = reinterpret_cast<const f32x4*>(smem + ((g - 1) * P::kW + in) * kOwn);
#pragma unroll
      for (int i = 0; i < P::kM; ++i)
#pragma unroll
        for (int j = 0; j < P::kT; ++j) acc[i][j] += from[(i * P::kT + j) * 64 + lane];
    }
  }
  return true;
}

// A wave's rows of results to memory in whole rows, through LDS of its own (16 rows of 32 BLOCKS bytes): BLOCKS
// blocks of 16 columns of each of 16 rows.  dst: the first row's first column; value(i, e): entry e of block i of
// these rows; rows before `from`, from n_rows on and columns from n_cols on are not written.
template <class T, int BLOCKS, class Value>
__device__ __forceinline__ void store_rows16(uint16_t* dst, int64_t ld, int64_t n_rows, int n_cols,
                                             unsigned char* own, int lane, Value&& value, int64_t from = 0) {
  constexpr int kRow = 32 * BLOCKS, kCh = kRow / 16, kPer = 64 / kCh;  // bytes, chunks; rows of a wave store
  const int r0 = lane & 15, q = lane >> 4;
  __atomic_signal_fence(__ATOMIC_SEQ_CST);  // (a wave's LDS operations execute in program order)
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i)
    *reinterpret_cast<uint2*>(own + r0 * kRow + (((2 * i + (q >> 1)) ^ (r0 % kCh)) << 4) + 8 * (q & 1)) =
        uint2{T::pack(value(i, 0), value(i, 1)), T::pack(value(i, 2), value(i, 3))};
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
  for (int k = 0; k < (16 + kPer - 1) / kPer; ++k) {
    const int r = k * kPer + lane / kCh, c = (lane % kCh) ^ (r % kCh);
    if (kPer > 16 && r >= 16) continue;
    const u32x4 v = *reinterpret_cast<const u32x4*>(own + r * kRow + (lane % kCh) * 16);
    if (r >= from && r < n_rows && 8 * c < n_cols) *reinterpret_cast<u32x4*>(dst + (int64_t)r * ld + 8 * c) = v;
  }
}

// A wave's rows of results to memory in whole rows, through LDS of its own: BLOCKS blocks of 32 columns of
// each of 32 rows at a time.  dst: the first row's first column; value(i, r): entry r of block i of these
// rows; rows from n_rows on and columns from n_cols on are not written.
template <class T, int BLOCKS, class Value>
__device__ __forceinline__ void store_rows(uint16_t* dst, int64_t ld, int64_t n_rows, int n_cols,
                                           unsigned char* own, int lane, Value&& value) {
  constexpr int kRow = 64 * BLOCKS;                             // bytes of a row
  constexpr int kCh = kRow / 16, kPer = 64 / kCh;               // chunks of a row, rows of a wave store
  const int half = lane >> 5, col = lane & 31;
  __atomic_signal_fence(__ATOMIC_SEQ_CST);  // (a wave's LDS operations execute in program order)
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2*>(own + col * kRow + (((4 * i + g) ^ (col % kCh)) << 4) + 8 * half) =
          uint2{T::pack(value(i, 4 * g), value(i, 4 * g + 1)), T::pack(value(i, 4 * g + 2), value(i, 4 * g + 3))};
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
  for (int k = 0; k < 32 / kPer; ++k) {
    const int r = k * kPer + lane / kCh, c = (lane % kCh) ^ (r % kCh);
    const u32x4 v = *reinterpret_cast<const u32x4*>(own + r * kRow + (lane % kCh) * 16);
    if (r < n_rows && 8 * c < n_cols) *reinterpret_cast<u32x4*>(dst + (int64_t)r * ld + 8 * c) = v;
  }
}

}  // namespace hpr
