// LDS tiles of 16-bit rows and their readers, and the search for a workgroup's sequence: shared by
// the encoder's operators.
#pragma once

#include "common.h"

namespace hpr {

// LDS tiles of `rows` rows of D 16-bit values: the 16-byte chunk c of row r is stored at position
// c ^ swz(r) of its row.  LDS serves 256 bytes (64 banks) a cycle.  row_frag reads one chunk of 16
// consecutive rows a cycle: swz, with the row's own offset at D = 64, spreads them over all 16
// positions.  tr_frag reads 64 bytes of four consecutive rows a cycle: the swizzle's upper bits, with
// that offset, send the four rows to the four quarters of the banks.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D >= 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// The same of rows of 64 values that are read 16 at a time, each in the four chunks of half a row by lanes 16 apart
// (operands of 16x16x32 products).  Of such a read LDS serves in a cycle rows 0-3 and 12-15 of one chunk with rows 4-11
// of its neighbour: with swz, which is for 32 rows of one chunk, each would take two (3 million cycles of conflicts in
// 13,063 rows, 4096 -> 14336, with swz 291 million, half of the reads' time).
__device__ __forceinline__ int swz16(int r) { return (r >> 1) & 7; }

// Offsets of a lane's reads from an LDS tile.
template <int D>
struct TileReads {
  int row0;              // row (lane & 31), byte offset
  int chunk0;            // 16 * (half ^ swz)
  int tr0;               // row of tr_frag, byte offset
  int trc;               // its chunk for d block 0, as byte offset, and the byte in the chunk
  __device__ __forceinline__ explicit TileReads(int lane) {
    const int r = lane & 31, half = lane >> 5;
    row0 = r * D * 2;
    chunk0 = (half ^ swz<D>(r)) << 4;
    const int i = lane & 15, e = i >> 2;
    const int tr = 4 * half + e;
    tr0 = tr * D * 2;
    trc = (((2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) ^ swz<D>(tr)) << 4) | ((i & 1) << 3);
  }
  // A copy whose addresses are formed where they are used.  Loop-invariant, a tile's 16 addresses would be
  // kept in registers, which kernels at their limit need to read operands ahead of the products.
  __device__ __forceinline__ TileReads fresh() const {
    TileReads r = *this;
    asm volatile("" : "+v"(r.chunk0), "+v"(r.trc));
    return r;
  }
  // Rows [32 blk, 32 blk + 32), values [16 s, 16 s + 16): the left operand of a product over d.
  __device__ __forceinline__ u32x4 row_frag(const unsigned char* tile, int blk, int s) const {
    return *reinterpret_cast<const u32x4*>(tile + blk * 32 * D * 2 + row0 + (chunk0 ^ (s << 5)));
  }
  // Columns [32 db, 32 db + 32) of rows [32 blk + 16 s, + 16): the left operand of a product over
  // rows, whose k follows the register order of a result: element e of half h is row
  // 8 (e / 4) + 4 h + e % 4.
  __device__ __forceinline__ u32x4 tr_frag(const unsigned char* tile, int blk, int s, int db) const {
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    typedef uint32_t v2u __attribute__((ext_vector_type(2)));
    const unsigned char* p = tile + (32 * blk + 16 * s) * D * 2 + tr0;
    const int c = trc ^ (db << 6);
    const v2u a = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + c)));
    const int c1 = c ^ 32;  // rows 8 further: bit 1 of swz
    const v2u b = __builtin_bit_cast(
        v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p + 8 * D * 2 + c1)));
    return u32x4{a[0], a[1], b[0], b[1]};
  }
};

__device__ __forceinline__ void sync_lds() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// Loads from global memory straight into LDS, 16 (or 4) bytes per lane at lds + 16 (4) lane, of kernels
// that read LDS by columns.  The compiler takes ds_read_b64_tr_b16 to depend on every such load that it
// knows of, and waits for the next stage's in the middle of this one's products (attention over 216
// sequences of about 250 tokens: 281 us, as written here 266 us).  So these are known to the program
// alone: it waits for them (s_waitcnt vmcnt) before the barrier that hands the stage over.  They have
// no output register, and the compiler's own counts of outstanding loads only become stricter.
typedef u32x4 rsrc_t;  // a raw buffer of 2^31 - 1 bytes from base
__device__ __forceinline__ rsrc_t rsrc_of(const void* base) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  return rsrc_t{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
}
// The LDS address of a __shared__ array (of the array itself: a generic pointer would need a check).
#define LDS_ADDRESS(array) ((uint32_t)(uintptr_t)(lds_void_t*)(array))
__device__ __forceinline__ void load_lds16(rsrc_t r, uint32_t lds, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(r)
               : "memory");
}
// The same without a place in the caches, for what is read once.
__device__ __forceinline__ void load_lds16_stream(rsrc_t r, uint32_t lds, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(r)
               : "memory");
}
__device__ __forceinline__ void load_lds16(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src)
               : "memory");
}
__device__ __forceinline__ void load_lds4(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src)
               : "memory");
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, 0x7fffffff,
                                           0x00020000);
}

// Loads a tile of ROWS rows of D values straight into LDS, NW waves sharing it: every wave load
// fills 1 KiB.  Rows past the last valid one repeat it, chunks past the row's `chunks` repeat the
// last (the products' other operand is zero there).
template <int D, int ROWS, int NW, bool BY16 = false>
struct TileLoad {
  static constexpr int kCh = D / 8;                       // chunks of a row
  static constexpr int kRows = 64 / kCh;                  // rows of a wave load
  static constexpr int kLoads = ROWS * kCh / 64 / NW;     // loads per wave
  static_assert(ROWS * kCh % (64 * NW) == 0, "a tile splits evenly over the waves");
  int row[kLoads], chunk[kLoads];                         // per lane
  __device__ __forceinline__ TileLoad(int wave, int lane, int chunks) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      row[j] = (wave * kLoads + j) * kRows + lane / kCh;
      const int c = (lane % kCh) ^ (BY16 ? swz16(row[j]) : swz<D>(row[j]));
      chunk[j] = (c < chunks ? c : chunks - 1) * 16;
    }
  }
};

// The last s in [0, n) with off[s] / ts + s <= tile (0 if none).  The whole wave searches.  (Rows are
// below 2^31; offsets that are not give some s.)
__device__ __forceinline__ int find_seq(const int64_t* off, int n, int ts, uint32_t tile) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int i = lane * step;
    const bool ok = i < n && (uint32_t)off[lo + i] / (uint32_t)ts + (uint32_t)(lo + i) <= tile;
    const unsigned long long b = __ballot(ok);
    int c = __popcll(b);
    c = c < 1 ? 1 : c;
    lo += (c - 1) * step;
    const int left = n - (c - 1) * step;
    n = step < left ? step : left;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The last s in [0, n) with off[s] <= row (0 if none).  The whole wave searches.
__device__ __forceinline__ int find_row(const int64_t* off, int n, int64_t row) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int i = lane * step;
    int c = __popcll(__ballot(i < n && off[lo + i] <= row));
    c = c < 1 ? 1 : c;
    lo += (c - 1) * step;
    const int left = n - (c - 1) * step;
    n = step < left ? step : left;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace hpr
