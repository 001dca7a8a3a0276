// Attention over packed sequences with grouped heads: forward, gradients, and the join of calls
// whose keys are split over workgroups.
//
// Sequence s holds query rows [q_off[s], q_off[s+1]) and key rows [k_off[s], k_off[s] + its key
// count).  For query head h, its kv head h / G, token i of lq and key j of lk:
//   visible(i, j):  j <= i + lk - lq (causal), j > i + lk - lq - window (window > 0)
//   x_ij = scale <q_i, k_j>,  p_ij = softmax of x_i. over the visible keys,  o_i = sum_j p_ij v_j
//   lse_i = log sum_j exp(x_ij)   (no visible key: o_i = 0, lse_i = -inf, no gradient)
// and with g = dL/do, delta_i = <g_i, o_i>, ds_ij = p_ij (<g_i, v_j> - delta_i):
//   dv_j = sum_i p_ij g_i,  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i
// with the sums for a kv head over all query heads of its group.
//
// Slots.  The query rows of a kv head's whole group share its keys, so a tile's rows are (token,
// head of the group) pairs, "slots": slot = token * G + head.  A tile takes TS = rows / G whole
// tokens.  Sequence s owns the tile numbers from q_off[s] / TS + s, which leaves every sequence at
// least ceil(lq / TS) of them (numbers past the sequence's end are no tiles).  In small calls a
// workgroup searches the offsets for its tile; calls of many tiles have a first launch write
// them down (plan_kernel).
//
// Products.  All of them are v_mfma_f32_32x32x16 with the 32 rows that a wave owns as the columns
// of the result, so a lane holds 16 entries of one of its rows (the entries of the two half-waves
// interleave by fours).  Row statistics are then per lane, and such a result, rounded to 16 bits,
// is the right operand of the next product as it stands: the left operand follows its order of k
// (see tr_frag).  Left operands are tiles in LDS, read by rows (row_frag) or by columns (tr_frag,
// ds_read_b64_tr_b16).
#include "common.h"
#include "half.h"
#include "kernels.h"
#include "tiles.h"

namespace hpr {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Stands for the maximum of no key yet, finite so that differences with it stay numbers.
constexpr float kNoMax = -1e30f;
// A row's running maximum is raised only when a score passes it by this much (in powers of two):
// the exponentials then stay below 2^8, harmless in fp32 sums and 16-bit products alike (their
// relative rounding does not depend on it), and most tiles skip the rescaling of the output.
constexpr float kRaise = 8.f;
// fp16 keeps fewer bits below 2^-14 and none below 2^-25, which is where the many keys of a row lie beside one that
// takes most of the attention: there the reference stays this much below the maximum, and the exponentials of a
// row reach from 2^15 down.
template <class T>
constexpr float kBelow = T::kNarrow ? 7.f : 0.f;

constexpr int kKeys = 64;  // keys per tile of the dq kernel

// max / sum over the two half-waves, in both of them
__device__ __forceinline__ float half_max(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

struct Seq {
  int64_t q0, k0;  // first rows
  int lq, lk;
};

// Bounds of sequence s, inside the tensors whatever the offsets hold.
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int s) {
  Seq r;
  auto clamp = [](int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); };
  r.q0 = clamp(a.q_off[s], 0, a.n_q);
  r.lq = (int)(clamp(a.q_off[s + 1], r.q0, a.n_q) - r.q0);
  r.k0 = clamp(a.k_off[s], 0, a.n_k);
  int64_t lk = clamp(a.k_off[s + 1], r.k0, a.n_k) - r.k0;
  if (a.k_len) lk = clamp(a.k_len[s], 0, lk);
  r.lk = (int)lk;
  return r;
}

// Tile `tile` of ts tokens a tile.  The whole wave searches.
__device__ __forceinline__ AttnTile find_q_tile(const AttnArgs& a, uint32_t tile, int ts) {
  const int s = find_seq(a.q_off, a.n_seq, ts, tile);
  const Seq S = seq_of(a, s);
  AttnTile r = {S.q0, S.k0, S.lq, S.lk, 0, 0};
  const int64_t first = ((int64_t)tile - ((uint32_t)S.q0 / (uint32_t)ts + (uint32_t)s)) * ts;
  if (first >= 0 && first < S.lq) {
    r.first = (int)first;
    r.n = S.lq - r.first < ts ? S.lq - r.first : ts;
  }
  return r;
}
// The same for tiles of `rows` key rows; the gradients' rows of a sequence are its whole room.
__device__ __forceinline__ AttnTile find_k_tile(const AttnArgs& a, uint32_t tile, int rows) {
  const int s = find_seq(a.k_off, a.n_seq, rows, tile);
  const Seq S = seq_of(a, s);
  AttnTile r = {S.q0, S.k0, S.lq, S.lk, 0, 0};
  const int64_t end = a.k_off[s + 1] < a.n_k ? a.k_off[s + 1] : a.n_k;
  const int64_t room = end - S.k0;
  const int64_t first = ((int64_t)tile - ((uint32_t)S.k0 / (uint32_t)rows + (uint32_t)s)) * rows;
  if (first >= 0 && first < room) {
    r.first = (int)first;
    r.n = room - first < rows ? (int)(room - first) : rows;
  }
  return r;
}
__device__ __forceinline__ AttnTile uniform_tile(const AttnTile* p) {
  AttnTile r = *p;  // (a uniform address: scalar loads)
  return r;
}

// Token of a tile's slot (a slot of at most 128).
__device__ __forceinline__ int token_of(const AttnArgs& a, int slot) {
  return (int)((uint32_t)slot * a.g_inv >> 16);
}

// Keys [lo, hi) visible from token i (of lq, with lk keys).
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, const AttnTile& s, int i) {
  Span r = {0, s.lk};
  if (a.causal) {
    const int64_t reach = (int64_t)i + s.lk - s.lq;  // the last visible key
    r.hi = reach < 0 ? 0 : (int)reach + 1;
    if (a.window > 0) {
      const int64_t lo = reach - a.window + 1;
      r.lo = lo < 0 ? 0 : (int)lo;
    }
  }
  return r;
}

// A wave's own 32 rows through its own 32 * D * 2 bytes of LDS, so that memory sees whole rows (by
// lanes a row's pieces of 16 or 32 bytes would be requests of their own).
template <int D>
struct WaveRows {
  static constexpr int kCh = D / 8, kRows = 64 / kCh, kLoads = 32 / kRows;
  static constexpr int kBytes = 32 * D * 2;
  // at(r): the byte offset of row r of the 32 from the buffer's base
  template <class F>
  static __device__ __forceinline__ void load(rsrc_t from, F at, uint32_t lds, int lane, int chunks) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRows + lane / kCh;
      const int c = (lane % kCh) ^ swz<D>(r);
      load_lds16(from, lds + j * 1024, at(r) + 16 * (c < chunks ? c : chunks - 1));
    }
  }
  // the loaded rows as right operands, zero past dim
  static __device__ __forceinline__ void cols(const TileReads<D>& rd, const unsigned char* lds, int dim,
                                              int half, u32x4 (&f)[D / 16]) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f[s] = rd.row_frag(lds, 0, s);
    if (dim < D) {
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        if (16 * s + 8 * half >= dim) f[s] = u32x4{0u, 0u, 0u, 0u};
    }
  }
  // the rows' chunks past dim become zero
  static __device__ __forceinline__ void clear(unsigned char* lds, int lane, int chunks) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRows + lane / kCh;
      if (((lane % kCh) ^ swz<D>(r)) >= chunks)
        *reinterpret_cast<u32x4*>(lds + j * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
    }
  }
  // x, times the lane's factor, as 16-bit rows: row r goes to byte offset at(r) from base if r < n
  template <class T, class F>
  static __device__ __forceinline__ void store(const f32x16 (&x)[D / 32], float factor, uint16_t* base,
                                               F at, int n, unsigned char* lds, int lane, int chunks) {
    const int row = lane & 31, half = lane >> 5;
    __atomic_signal_fence(__ATOMIC_SEQ_CST);  // (a wave's LDS operations execute in program order)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(lds + row * D * 2 + (((4 * db + g) ^ swz<D>(row)) << 4) + 8 * half) =
            uint2{T::pack(x[db][4 * g] * factor, x[db][4 * g + 1] * factor),
                  T::pack(x[db][4 * g + 2] * factor, x[db][4 * g + 3] * factor)};
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    const int last = n - 1 < 31 ? n - 1 : 31;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRows + lane / kCh;
      const int c = (lane % kCh) ^ swz<D>(r);
      const u32x4 v = *reinterpret_cast<const u32x4*>(lds + j * 1024 + lane * 16);
      if (r <= last && c < chunks)
        *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(base) + (uint32_t)(at(r) + 16 * c)) = v;
    }
  }
};

// The slots of a wave, as byte offsets from their tile's first token: row r of the 32 is slot
// first + r (the last slot past it), token slot / G of the tile, head slot % G of the group.
struct SlotRows {
  uint32_t first, last, g_inv, step, head;  // step: a token's bytes less G heads', head: a head's
  __device__ __forceinline__ SlotRows(const AttnArgs& a, int wave, int n_slot, int64_t row, int64_t head_)
      : first(wave * 32),
        last(n_slot - 1),
        g_inv(a.g_inv),
        step((uint32_t)(row - a.G * head_) * 2u),
        head((uint32_t)head_ * 2u) {}
  // (token * row + (slot - token * G) * head, in 32-bit arithmetic that wraps and comes back)
  __device__ __forceinline__ uint32_t operator()(int r) const {
    const uint32_t s = first + r < last ? first + r : last;
    return ((s * g_inv) >> 16) * step + s * head;
  }
};

// A stage's loads: KEYS rows of K, then of V, straight into LDS.  The offsets of a whole tile are
// kept per lane; the sequence's last tile forms its own, and so does the one where a window begins:
// keys that no query sees may hold anything, and their probability of 0 would keep a NaN or an infinity.
template <int D, int NW, int KEYS, bool STREAM = false>
struct KvLoad {
  using L = TileLoad<D, KEYS, NW>;
  L at;
  const uint16_t *k, *v;  // the kv head's first rows
  int ok[L::kLoads], ov[L::kLoads];
  __device__ __forceinline__ KvLoad(const AttnArgs& a, const AttnTile& S, int kvh, int wave, int lane)
      : at(wave, lane, a.dim / 8),
        k(a.k + S.k0 * a.k_row + kvh * a.k_head),
        v(a.v + S.k0 * a.v_row + kvh * a.v_head) {
#pragma unroll
    for (int j = 0; j < L::kLoads; ++j) {
      ok[j] = at.row[j] * (int)a.k_row * 2 + at.chunk[j];
      ov[j] = at.row[j] * (int)a.v_row * 2 + at.chunk[j];
    }
  }
  static __device__ __forceinline__ void load(rsrc_t r, uint32_t lds, uint32_t offset) {
    if constexpr (STREAM)
      load_lds16_stream(r, lds, offset);
    else
      load_lds16(r, lds, offset);
  }
  __device__ __forceinline__ void issue(const AttnArgs& a, const AttnTile& S, uint32_t st, int wave,
                                        int kt, int lo) const {
    const int first = kt * KEYS;
    const int last = S.lk - 1 - first;  // last valid row of the tile (>= 0)
    const int low = lo - first;         // its first row that a query sees (<= last)
    const rsrc_t rk = rsrc_of(k + (int64_t)first * a.k_row);
    const rsrc_t rv = rsrc_of(v + (int64_t)first * a.v_row);
    const uint32_t to = st + wave * L::kLoads * 1024;  // LDS address
    constexpr int kTile = KEYS * D * 2;
    if (last >= KEYS - 1 && low <= 0) {
#pragma unroll
      for (int j = 0; j < L::kLoads; ++j) load(rk, to + j * 1024, ok[j]);
#pragma unroll
      for (int j = 0; j < L::kLoads; ++j) load(rv, to + kTile + j * 1024, ov[j]);
    } else {
#pragma unroll
      for (int j = 0; j < L::kLoads; ++j) {
        const int up = at.row[j] > low ? at.row[j] : low, r = up < last ? up : last;
        load(rk, to + j * 1024, r * (int)a.k_row * 2 + at.chunk[j]);
        load(rv, to + kTile + j * 1024, r * (int)a.v_row * 2 + at.chunk[j]);
      }
    }
  }
};

// A probability from the logarithm (base 2) of it.  An fp32 lse of enormous scores is off by more than
// a power of two; the clamp (an output modifier, free) keeps such rows finite.
__device__ __forceinline__ float prob(float x) {
  return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f);
}

// ds and p as operands of fp16 calls.  Below 2^-14 fp16 keeps fewer bits and below 2^-25 none, and that is
// where they lie for long rows and for small gradients (2,048 keys, dout of 1e-5: dq was off by 23 %, as
// rounding ds alone makes it).  So a lane's column of ds is held times a power of two, by which the sums are
// divided in the end: lowered, and the sums so far with it, where the column would pass 2^15, so that its
// largest entry is then in [2^9, 2^10).  p, which is at most 1, is held times 2^15.  The forward
// and the gradients take 3 to 5 % longer for it: 128 documents of up to 512 tokens, 12 heads of 64, 265 us (253;
// dq 87 and 82, dk/dv 119 and 109), 4 of 4,000 both ways 1,043 (989).
constexpr float kDsFrom = 0x1p60f;  // products of three fp16 sums stay finite
constexpr float kDsMost = 0x1p15f, kPScale = 0x1p15f;
template <int N>
__device__ __forceinline__ void keep_range(f32x16& ds, f32x16 (&sum)[N], float& factor) {
  float top = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) top = fmaxf(top, __builtin_fabsf(ds[r]));
  top = half_max(top);
  if (!__any(top > kDsMost)) return;
  const float by =
      top > kDsMost ? __builtin_amdgcn_ldexpf(1.f, 10 - __builtin_amdgcn_frexp_expf(top)) : 1.f;
  factor *= by;
#pragma unroll
  for (int r = 0; r < 16; ++r) ds[r] *= by;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[i][r] *= by;
}

// Scheduling groups: the next n LDS reads / products of the region go here.
#define sched_ds(n) __builtin_amdgcn_sched_group_barrier(0x100, n, 0)
#define sched_mfma(n) __builtin_amdgcn_sched_group_barrier(0x008, n, 0)

// ---- forward --------------------------------------------------------------------------------

// One tile of NW * 32 slots of one kv head against a split of its visible keys, KEYS at a time
// through NST LDS stages: one pass with the running maximum and sum of the softmax (fp32) in registers.
// Probabilities are rounded to 16 bits as the operand of the product with v, the output once.
//
// Measured, 32 heads of 128 on 8 kv heads, causal: one sequence of 32,768 tokens 7.9-8.3 ms from card to card,
// 1.06-1.12 PFLOP/s of the visible pairs, the matrix cores busy 59 % of the cycles at the 1.7 GHz that the
// card's power limit leaves on random operands (zeros run in 5.9-6.8 ms).  256 sequences of 32 to 384 tokens
// 0.25-0.26 ms, where q, k, v and the output, the whole of its traffic, take 0.16 ms of HBM: a workgroup lives
// for 4.7 stages on average, so that its start and end are seen (matrix cores busy 23 %, vector instructions 41
// % of the cycles; 87 % of the pairs that the waves compute are visible).  A token of each of 64 caches of up to
// 8,192 keys 185-190 us and 5 us for the join, 6.1 TB/s of keys and values.
template <class T, int D, int NW, int KEYS, int NST>
__device__ __forceinline__ void attn_fwd(const AttnArgs& a) {
  constexpr int kS = D / 16, kDb = D / 32;
  constexpr int kB = KEYS / 32;
  constexpr int kTile = KEYS * D * 2;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NST * 2 * kTile];
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups are dealt to the XCDs in turn.  With several waves a workgroup, heads go round first:
  // the tiles of a head meet in one L2.  Single waves read every key once: there the heads of a run
  // of keys go to one XCD, one after another, so that it reads whole rows.
  uint32_t kvh, w;
  if constexpr (NW > 1) {
    kvh = blockIdx.x % (uint32_t)a.kv_heads;
    w = blockIdx.x / (uint32_t)a.kv_heads;
  } else {
    kvh = (blockIdx.x >> 3) % (uint32_t)a.kv_heads;
    w = (blockIdx.x >> 3) / (uint32_t)a.kv_heads * 8 + (blockIdx.x & 7);
    if (w >= (uint32_t)(a.tiles * a.splits)) return;
  }
  const int split = a.splits > 1 ? w % (uint32_t)a.splits : 0;
  // late tiles see the most keys: first
  const uint32_t tile = (uint32_t)a.tiles - 1 - (a.splits > 1 ? w / (uint32_t)a.splits : w);
  const AttnTile S = a.q_plan ? uniform_tile(a.q_plan + tile) : find_q_tile(a, tile, a.ts);
  if (S.n == 0) return;
  const int t0 = S.first, n_tok = S.n;

  // this lane's slot
  const int slot = wave * 32 + col;
  const int n_slot = n_tok * a.G;
  const bool live = slot < n_slot;
  const bool wave_live = wave * 32 < n_slot;
  const int cs = live ? slot : n_slot - 1;
  const int tok = t0 + token_of(a, cs), head = kvh * a.G + cs - token_of(a, cs) * a.G;
  const Span mine = span_of(a, S, tok);
  const int last_slot = wave * 32 + 31 < n_slot ? wave * 32 + 31 : n_slot - 1;
  const Span wfirst = span_of(a, S, t0 + token_of(a, wave_live ? wave * 32 : 0));
  const Span wlast = span_of(a, S, t0 + token_of(a, last_slot));
  const Span tfirst = span_of(a, S, t0), tlast = span_of(a, S, t0 + n_tok - 1);

  // key tiles of this split
  const int k_first = tfirst.lo / KEYS, k_end = (tlast.hi + KEYS - 1) / KEYS;
  const int n_kt = k_end > k_first ? k_end - k_first : 0;
  int kt0 = k_first, kt1 = k_first + n_kt;
  if (a.splits > 1) {  // (below 2^26 tiles, times 64)
    kt0 = k_first + (int)((uint32_t)n_kt * (uint32_t)split / (uint32_t)a.splits);
    kt1 = k_first + (int)((uint32_t)n_kt * (uint32_t)(split + 1) / (uint32_t)a.splits);
  }

  const KvLoad<D, NW, KEYS, NW == 1> ld(a, S, kvh, wave, lane);
  auto issue = [&](int buf, int kt) {
    ld.issue(a, S, LDS_ADDRESS(smem) + buf * 2 * kTile, wave, kt, tfirst.lo);
  };
  // q through the later stages, which the loop fills only after its first barrier
  static_assert(NW * WaveRows<D>::kBytes <= (NST - 1) * 2 * kTile, "the waves' rows fit there");
  unsigned char* own = smem + 2 * kTile + wave * WaveRows<D>::kBytes;
  WaveRows<D>::load(rsrc_of(a.q + (S.q0 + t0) * a.q_row + kvh * a.G * a.q_head),
                    SlotRows(a, wave, n_slot, a.q_row, a.q_head),
                    LDS_ADDRESS(smem) + 2 * kTile + wave * WaveRows<D>::kBytes, lane, a.dim / 8);
  if (kt0 < kt1) {
    issue(0, kt0);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * ld.at.kLoads));
  } else {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  }
  const TileReads<D> rd(lane);
  u32x4 q[kS];
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  WaveRows<D>::cols(rd, own, a.dim, half, q);

  f32x16 o[kDb];
#pragma unroll
  for (int db = 0; db < kDb; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  float m = kNoMax, l = 0.f;

#pragma unroll 1
  for (int kt = kt0, buf = 0; kt < kt1; ++kt, buf = buf + 1 < NST ? buf + 1 : 0) {
    if (NST == 2 || kt == kt0 || kt + 1 == kt1)
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    else  // the next tile may be on its way
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * ld.at.kLoads));
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    sync_lds();  // the tile has landed, and nobody reads the stage before it any more
    if (NST == 2) {
      if (kt + 1 < kt1) issue(buf ^ 1, kt + 1);
    } else {
      if (kt == kt0 && kt + 1 < kt1) issue(1, kt + 1);
      if (kt + 2 < kt1) issue(buf == 0 ? 2 : buf - 1, kt + 2);
    }
    const int first = kt * KEYS;
    if (!wave_live || first >= wlast.hi || first + KEYS <= wfirst.lo) continue;
    const unsigned char* ks = smem + buf * 2 * kTile;
    const unsigned char* vs = ks + kTile;
    f32x16 x[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[b][r] = 0.f;
#pragma unroll
    for (int s = 0; s < kS; ++s)
#pragma unroll
      for (int b = 0; b < kB; ++b) x[b] = T::mfma(rd.row_frag(ks, b, s), q[s], x[b]);
    // the operands' reads run two k-steps ahead of the products
    sched_ds(2 * kB);
#pragma unroll
    for (int s = 0; s < kS - 2; ++s) {
      sched_mfma(kB);
      sched_ds(kB);
    }
    sched_mfma(2 * kB);
    __builtin_amdgcn_sched_barrier(0);
    if (first + KEYS > wfirst.hi) {  // some key is past some slot's last
      const int hi = mine.hi - first - 4 * half;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * b + 8 * (r >> 2) + (r & 3) >= hi) x[b][r] = -__builtin_inff();
    }
    if (first < wlast.lo) {  // or before some slot's first
      const int lo = mine.lo - first - 4 * half;
#pragma unroll
      for (int b = 0; b < kB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * b + 8 * (r >> 2) + (r & 3) < lo) x[b][r] = -__builtin_inff();
    }
    float top = x[0][0];
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[b][r]);
    top = half_max(top) * a.c;
    if (__any(top > m + (kRaise + kBelow<T>))) {
      const float mn = fmaxf(m, top - kBelow<T>);
      const float f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int db = 0; db < kDb; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= f;
    }
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      u32x4 p[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][r], a.c, -m));
        l += x[b][r];
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[s][e] = T::pack(x[b][8 * s + 2 * e], x[b][8 * s + 2 * e + 1]);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int db = 0; db < kDb; ++db) o[db] = T::mfma(rd.tr_frag(vs, b, s, db), p[s], o[db]);
    }
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  l = half_sum(l);
  const int64_t row = (S.q0 + tok) * a.heads + head;
  if (a.splits > 1) {
    // unnormalised sums, their reference maximum and total: attn_join_kernel
    if (!live) return;
    const int64_t at = ((int64_t)split * a.n_q * a.heads + row);
    float* dst = a.part_o + at * a.dim;
#pragma unroll
    for (int db = 0; db < kDb; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * db + 8 * g + 4 * half;
        if (d < a.dim)
          *reinterpret_cast<f32x4*>(dst + d) =
              f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
      }
    if (half == 0) {
      a.part_ml[2 * at] = m;
      a.part_ml[2 * at + 1] = l;
    }
    return;
  }
  if (a.lse && live && half == 0) a.lse[row] = l > 0.f ? (m + log2f(l)) * kLn2 : -__builtin_inff();
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  sync_lds();  // nobody reads the stages any more
  WaveRows<D>::template store<T>(o, l > 0.f ? 1.f / l : 0.f,
                                 a.out + ((S.q0 + t0) * a.heads + kvh * a.G) * a.dim,
                                 SlotRows(a, wave, n_slot, (int64_t)a.heads * a.dim, a.dim),
                                 n_slot - wave * 32, own, lane, a.dim / 8);
}

// out = the splits' sums joined under their common maximum.  A wave per (token, head): lane s holds
// split s's statistics, then lane i values 2 i and 2 i + 1.  Bound by the latency of its two loads: 4.9 us
// for 64 tokens of 32 heads of 128 in 8 splits (8 MB).
constexpr int kMaxSplits = 64;
static_assert(kMaxSplits <= 64 && kMaxSplits % 4 == 0, "a lane per split, four splits a step");

template <class T>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  const int64_t rows = a.n_q * a.heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  float2 ml = {kNoMax, 0.f};
  if (lane < a.splits) ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (lane * rows + row));
  const float m = wave_max(ml.x);
  const float f = lane < a.splits ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
  const float l = wave_sum(f * ml.y);
  const int d = 2 * lane < a.dim ? 2 * lane : 0;
  const float* src = a.part_o + row * a.dim + d;
  float o0 = 0.f, o1 = 0.f;
  for (int s0 = 0; s0 < a.splits; s0 += 4) {  // four loads together, the last split again past the end
    float2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = s0 + i < a.splits ? s0 + i : a.splits - 1;
      v[i] = *reinterpret_cast<const float2*>(src + s * rows * a.dim);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s0 + i));
      o0 += fs * v[i].x;
      o1 += fs * v[i].y;
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (2 * lane < a.dim)
    *reinterpret_cast<uint32_t*>(a.out + row * a.dim + d) = T::pack(o0 * inv, o1 * inv);
  if (a.lse && lane == 0) a.lse[row] = l > 0.f ? (m + log2f(l)) * kLn2 : -__builtin_inff();
}

// ---- gradients --------------------------------------------------------------------------------

// dq of a tile of slots, over all their visible keys; also delta (fp32), which the dk/dv kernel reads.
// ds is rounded to 16 bits as the operand of the product with k, dq once.  Where all the keys that a wave's
// rows see lie in one stage (of 64 keys from a multiple of 64 on), delta is summed from p and dp before ds is formed: of few keys, p (dp - delta)
// cancels, and the rounding of out would be seen in it (a row's first key alone: ds is 0).  On the documents
// below dq and dk were off by 2.5e-3 without that and are by 2.4e-3 (an exact result rounded to bf16: 1.7e-3),
// in the same time.  Two kernels, this and the dk/dv kernel, each with the sums of its own rows in
// registers: fused, one of the sums would go out through atomics, whose order changes results, or as fp32
// parts.
//
// Measured, 192 documents of 64 to 448 tokens and 24 questions, 32 heads of 128 on 8 kv heads, causal: 365-390
// us, bound by HBM (1.4 GB read and 0.4 written, 265 us) and by a workgroup's start (three dependent loads: q and dout, out, keys; two
// workgroups per CU); the matrix cores are busy 24 % of the cycles.  One sequence of 8,192 tokens: both kernels
// at 1.09 PFLOP/s of the visible pairs.
template <class T, int D, int NW>
__device__ __forceinline__ void attn_dq(const AttnArgs& a) {
  constexpr int kS = D / 16, kDb = D / 32;
  constexpr int kTile = kKeys * D * 2;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * kTile];
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % (uint32_t)a.kv_heads;
  const uint32_t tile = (uint32_t)a.tiles - 1 - blockIdx.x / (uint32_t)a.kv_heads;
  const AttnTile S = a.q_plan ? uniform_tile(a.q_plan + tile) : find_q_tile(a, tile, a.ts);
  if (S.n == 0) return;
  const int t0 = S.first, n_tok = S.n;
  const int slot = wave * 32 + col;
  const int n_slot = n_tok * a.G;
  const bool live = slot < n_slot;
  const bool wave_live = wave * 32 < n_slot;
  const int cs = live ? slot : n_slot - 1;
  const int tok = t0 + token_of(a, cs), head = kvh * a.G + cs - token_of(a, cs) * a.G;
  const Span mine = span_of(a, S, tok);
  const int last_slot = wave * 32 + 31 < n_slot ? wave * 32 + 31 : n_slot - 1;
  const Span wfirst = span_of(a, S, t0 + token_of(a, wave_live ? wave * 32 : 0));
  const Span wlast = span_of(a, S, t0 + token_of(a, last_slot));
  const Span tfirst = span_of(a, S, t0), tlast = span_of(a, S, t0 + n_tok - 1);
  const int kt0 = tfirst.lo / kKeys, kt1 = (tlast.hi + kKeys - 1) / kKeys;

  const int64_t row = (S.q0 + tok) * a.heads + head;
  const SlotRows dense(a, wave, n_slot, (int64_t)a.heads * a.dim, a.dim);
  const int64_t dense0 = ((S.q0 + t0) * a.heads + kvh * a.G) * a.dim;
  const KvLoad<D, NW, kKeys> ld(a, S, kvh, wave, lane);
  auto issue = [&](int buf, int kt) {
    ld.issue(a, S, LDS_ADDRESS(smem) + buf * 2 * kTile, wave, kt, tfirst.lo);
  };
  // q through the second stage, dout through the first, then out through the second
  constexpr int kOwn = WaveRows<D>::kBytes;
  static_assert(NW * kOwn <= 2 * kTile, "the wave's rows fit a stage");
  const TileReads<D> rd(lane);
  unsigned char* own = smem + 2 * kTile + wave * kOwn;
  const uint32_t own_at = LDS_ADDRESS(smem) + 2 * kTile + wave * kOwn;
  WaveRows<D>::load(rsrc_of(a.q + (S.q0 + t0) * a.q_row + kvh * a.G * a.q_head),
                    SlotRows(a, wave, n_slot, a.q_row, a.q_head), own_at, lane, a.dim / 8);
  WaveRows<D>::load(rsrc_of(a.dout + dense0), dense, LDS_ADDRESS(smem) + wave * kOwn, lane, a.dim / 8);
  const float lse2 = a.lse[row] * kLog2e;
  u32x4 q[kS], g[kS];
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  WaveRows<D>::cols(rd, own, a.dim, half, q);
  WaveRows<D>::cols(rd, smem + wave * kOwn, a.dim, half, g);
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  sync_lds();
  WaveRows<D>::load(rsrc_of(a.out + dense0), dense, own_at, lane, a.dim / 8);
  if (kt0 < kt1) {
    issue(0, kt0);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * ld.at.kLoads));
  } else {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  }
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  float delta = 0.f;
  {
    u32x4 o[kS];
    WaveRows<D>::cols(rd, own, a.dim, half, o);
#pragma unroll
    for (int s = 0; s < kS; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        delta += T::lo(g[s][e]) * T::lo(o[s][e]) + T::hi(g[s][e]) * T::hi(o[s][e]);
    delta = half_sum(delta);
  }

  f32x16 dq[kDb];
#pragma unroll
  for (int db = 0; db < kDb; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[db][r] = 0.f;
  float range = T::kNarrow ? kDsFrom : 1.f;  // of ds and dq (keep_range)

#pragma unroll 1
  for (int kt = kt0; kt < kt1; ++kt) {
    const int buf = (kt - kt0) & 1;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    sync_lds();
    if (kt + 1 < kt1) issue(buf ^ 1, kt + 1);
    const int first = kt * kKeys;
    if (!wave_live || first >= wlast.hi || first + kKeys <= wfirst.lo) continue;
    const unsigned char* ks = smem + buf * 2 * kTile;
    const unsigned char* vs = ks + kTile;
    // p and dp of 32 keys from `at`, the second or first half of the stage
    auto scores = [&](int b, int at, f32x16& x, f32x16& dp) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = 0.f, dp[r] = 0.f;
#pragma unroll
      for (int s = 0; s < kS; ++s) {
        x = T::mfma(rd.row_frag(ks, b, s), q[s], x);
        dp = T::mfma(rd.row_frag(vs, b, s), g[s], dp);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = prob(__builtin_fmaf(x[r], a.c, -lse2));
      if (at + 32 > wfirst.hi) {  // some key is past some slot's last
        const int hi = mine.hi - at - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) >= hi) x[r] = 0.f;
      }
      if (at < wlast.lo) {  // or before some slot's first
        const int lo = mine.lo - at - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) < lo) x[r] = 0.f;
      }
    };
    if (first <= wfirst.lo && wlast.hi <= first + kKeys) {
      delta = 0.f;
#pragma unroll 1
      for (int b = 0; b < 2; ++b) {
        if (first + 32 * b >= wlast.hi) break;
        f32x16 x, dp;
        scores(b, first + 32 * b, x, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) delta += x[r] * dp[r];
      }
      delta = half_sum(delta);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int at = first + 32 * b;
      if (at >= wlast.hi || at + 32 <= wfirst.lo) continue;
      f32x16 x, dp;
      scores(b, at, x, dp);
      u32x4 ds[2];
      if constexpr (T::kNarrow) {
        const float d = -delta * range;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] *= __builtin_fmaf(dp[r], range, d);
        keep_range(x, dq, range);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] *= dp[r] - delta;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) ds[s][e] = T::pack(x[8 * s + 2 * e], x[8 * s + 2 * e + 1]);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int db = 0; db < kDb; ++db) dq[db] = T::mfma(rd.tr_frag(ks, b, s, db), ds[s], dq[db]);
    }
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  if (live && half == 0) a.delta[row] = delta;
  if (!a.dq) return;
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  sync_lds();  // nobody reads the stages any more
  WaveRows<D>::template store<T>(dq, a.scale / range, a.dq + dense0, dense, n_slot - wave * 32, own, lane,
                                 a.dim / 8);
}

// dk and dv of a tile of NW * 32 keys of one kv head, over all the slots that see them, kSlots
// (whole tokens of G slots) at a time.  A wave owns 32 keys; the sum over the group's heads is
// the sum over slots.  The wave's K stays in registers, its V in LDS: with the 128 registers of both
// sums at D = 128, that is what leaves room for two waves per SIMD (one wave, with V in registers: 930 us
// on the documents of the dq kernel's comment, 390-415 us so).  Bound there as the dq kernel is (q and dout are
// read again for every 128 keys: 1.6 GB read and 0.2 written, 267 us of HBM; matrix cores 28 % busy).  128
// documents of up to 512 tokens, both ways, 12 heads of 64, fp16: 88 us (dq) and 118 us.
constexpr int kSlots = 32;

template <class T, int D, int NW>
__device__ __forceinline__ void attn_dkv(const AttnArgs& a) {
  constexpr int kS = D / 16, kDb = D / 32;
  constexpr int kTile = kSlots * D * 2;
  constexpr int kStage = 2 * kTile + 2 * 64 * 4;  // q, dout, lse, delta (a lane each, 32 used)
  constexpr int kOwn = WaveRows<D>::kBytes;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * kStage + NW * kOwn];
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % (uint32_t)a.kv_heads;
  const uint32_t tile = blockIdx.x / (uint32_t)a.kv_heads;  // early keys are seen by the most tokens: first
  const AttnTile S = a.k_plan ? uniform_tile(a.k_plan + tile) : find_k_tile(a, tile, NW * 32);
  if (S.n == 0) return;
  const int key0 = S.first;
  const int key = key0 + wave * 32 + col;
  const bool seen = key < S.lk;  // (the gradient rows past the key count get zeros)

  // tokens that see a key of the tile / of the wave: causal i >= key - (lk - lq), and with a
  // window i < key - (lk - lq) + window
  const int shift = S.lk - S.lq;
  auto first_tok = [&](int k) {
    const int t = a.causal ? k - shift : 0;
    return t < 0 ? 0 : t;
  };
  auto end_tok = [&](int k) {
    if (!(a.causal && a.window > 0)) return S.lq;
    const int64_t t = (int64_t)k - shift + a.window;
    return t < 0 ? 0 : (t < S.lq ? (int)t : S.lq);
  };
  const int kend = key0 + NW * 32 - 1 < S.lk - 1 ? key0 + NW * 32 - 1 : S.lk - 1;
  const int ts = a.ts;
  int st0 = 0, st1 = 0;  // stages of ts tokens
  if (key0 < S.lk) {
    st0 = first_tok(key0) / ts;
    st1 = (end_tok(kend) + ts - 1) / ts;
  }
  const int wk0 = key0 + wave * 32;
  const bool wave_live = wk0 < S.lk;
  const int wk1 = wk0 + 31 < S.lk - 1 ? wk0 + 31 : S.lk - 1;
  const int my_first = first_tok(key), my_end = seen ? end_tok(key) : 0;
  const int w_first = first_tok(wk0), w_end = end_tok(wk1);            // any of the wave's keys
  const int w_first_all = first_tok(wk1), w_end_all = end_tok(wk0);    // all of them

  const TileReads<D> rd0(lane);
  const TileLoad<D, kSlots, NW> ld(wave, lane, a.dim / 8);
  const int used = ts * a.G;  // slots of a stage
  int tok_of[ld.kLoads], q_at[ld.kLoads], g_at[ld.kLoads];
#pragma unroll
  for (int j = 0; j < ld.kLoads; ++j) {
    const int r = ld.row[j] < used ? ld.row[j] : used - 1;
    tok_of[j] = token_of(a, r);
    const int head = r - tok_of[j] * a.G;
    q_at[j] = head * (int)a.q_head * 2 + ld.chunk[j];
    g_at[j] = head * a.dim * 2 + ld.chunk[j];
  }
  const int lr = lane < used ? lane : used - 1;
  const int l_tok = token_of(a, lr), l_head = lr - l_tok * a.G;
  const int64_t d_row = (int64_t)a.heads * a.dim;
  const uint16_t* qb = a.q + S.q0 * a.q_row + kvh * a.G * a.q_head;
  const uint16_t* gb = a.dout + S.q0 * d_row + kvh * a.G * a.dim;
  const float* stat = (wave == 0 ? a.lse : a.delta) + S.q0 * a.heads + kvh * a.G + l_head;
  auto issue = [&](int buf, int st) {
    const int t = st * ts;
    const int last = S.lq - 1 - t;  // last valid token of the stage
    const rsrc_t rq = rsrc_of(qb + (int64_t)t * a.q_row);
    const rsrc_t rg = rsrc_of(gb + (int64_t)t * d_row);
    const uint32_t base = LDS_ADDRESS(smem) + buf * kStage;
#pragma unroll
    for (int j = 0; j < ld.kLoads; ++j) {
      const int tk = tok_of[j] < last ? tok_of[j] : last;
      load_lds16(rq, base + (wave * ld.kLoads + j) * 1024, tk * (int)a.q_row * 2 + q_at[j]);
      load_lds16(rg, base + kTile + (wave * ld.kLoads + j) * 1024, tk * a.heads * a.dim * 2 + g_at[j]);
    }
    if (wave < 2)  // statistics: wave 0 lse, wave 1 delta, a slot per lane
      load_lds4(stat + (int64_t)(t + (l_tok < last ? l_tok : last)) * a.heads,
                base + 2 * kTile + wave * 64 * 4);
  };

  // k, then v, through the wave's own rows of LDS, where v stays
  unsigned char* own = smem + 2 * kStage + wave * kOwn;
  const uint32_t own_at = LDS_ADDRESS(smem) + 2 * kStage + wave * kOwn;
  u32x4 k[kS];
#pragma unroll
  for (int s = 0; s < kS; ++s) k[s] = u32x4{0u, 0u, 0u, 0u};
  if (wave_live) {
    const int last = S.lk - 1 - wk0;  // the rows past it repeat it
    WaveRows<D>::load(rsrc_of(a.k + (S.k0 + wk0) * a.k_row + kvh * a.k_head),
                      [&](int r) { return (uint32_t)(r < last ? r : last) * (uint32_t)a.k_row * 2u; },
                      own_at, lane, a.dim / 8);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    WaveRows<D>::cols(rd0, own, a.dim, half, k);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    WaveRows<D>::load(rsrc_of(a.v + (S.k0 + wk0) * a.v_row + kvh * a.v_head),
                      [&](int r) { return (uint32_t)(r < last ? r : last) * (uint32_t)a.v_row * 2u; },
                      own_at, lane, a.dim / 8);
    if (a.dim < D) {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
      __atomic_signal_fence(__ATOMIC_SEQ_CST);
      WaveRows<D>::clear(own, lane, a.dim / 8);
    }
  }
  f32x16 dk[kDb], dv[kDb];
#pragma unroll
  for (int db = 0; db < kDb; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[db][r] = 0.f, dv[db][r] = 0.f;
  float range = T::kNarrow ? kDsFrom : 1.f;  // of ds and dk (keep_range)

  if (st0 < st1) issue(0, st0);
#pragma unroll 1
  for (int st = st0; st < st1; ++st) {
    const int buf = (st - st0) & 1;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    sync_lds();
    if (st + 1 < st1) issue(buf ^ 1, st + 1);
    const int t = st * ts;
    if (!wave_live || t >= w_end || t + ts <= w_first) continue;
    const unsigned char* qs = smem + buf * kStage;
    const unsigned char* gs = qs + kTile;
    const float* lse_s = reinterpret_cast<const float*>(qs + 2 * kTile);
    const float* del_s = lse_s + 64;
    // some slot's token comes before those that see some key of the wave, or after them (or is none)
    const bool before = t < w_first_all;
    const bool past = used < kSlots || t + ts > S.lq || t + ts > w_end_all || wk0 + 31 >= S.lk;
    const TileReads<D> rd = rd0.fresh();
    f32x16 x, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f, dp[r] = 0.f;
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      x = T::mfma(rd.row_frag(qs, 0, s), k[s], x);
      dp = T::mfma(rd.row_frag(gs, 0, s), rd.row_frag(own, 0, s), dp);
    }
    // the operands' reads run ahead of the products
    sched_ds(6);
#pragma unroll
    for (int s = 0; s < kS - 2; ++s) {
      sched_mfma(2);
      sched_ds(3);
    }
    sched_mfma(4);
    __builtin_amdgcn_sched_barrier(0);
    u32x4 p16[2], ds[2];
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x4 ls = *reinterpret_cast<const f32x4*>(lse_s + 8 * q4 + 4 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[4 * q4 + e] = prob(__builtin_fmaf(x[4 * q4 + e], a.c, -ls[e] * kLog2e));
    }
    // the lane's key is seen from slots [lo, hi) of the stage (dp of a key that no query sees may be NaN)
    if (before) {
      const int lo = (my_first - t) * a.G - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) < lo) x[r] = dp[r] = 0.f;
    }
    if (past) {
      int hi = (my_end - t) * a.G;
      hi = (hi < used ? hi : used) - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= hi) x[r] = dp[r] = 0.f;
    }
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const f32x4 dl = *reinterpret_cast<const f32x4*>(del_s + 8 * q4 + 4 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dp[4 * q4 + e] = x[4 * q4 + e] * (dp[4 * q4 + e] - dl[e]);
        if constexpr (T::kNarrow) dp[4 * q4 + e] *= range, x[4 * q4 + e] *= kPScale;
      }
    }
    if constexpr (T::kNarrow) keep_range(dp, dk, range);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p16[s][e] = T::pack(x[8 * s + 2 * e], x[8 * s + 2 * e + 1]);
        ds[s][e] = T::pack(dp[8 * s + 2 * e], dp[8 * s + 2 * e + 1]);
      }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < kDb; ++db) {
        dv[db] = T::mfma(rd.tr_frag(gs, 0, s, db), p16[s], dv[db]);
        dk[db] = T::mfma(rd.tr_frag(qs, 0, s, db), ds[s], dk[db]);
      }
    sched_ds(8);
#pragma unroll
    for (int i = 0; i < 2 * kDb - 2; ++i) {
      sched_mfma(2);
      sched_ds(4);
    }
    sched_mfma(4);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
  // (keys that the sequence does not count have no sums)
  const int64_t first = ((S.k0 + wk0) * a.kv_heads + kvh) * a.dim;
  auto at = [&](int r) { return (uint32_t)r * (uint32_t)(a.kv_heads * a.dim) * 2u; };
  WaveRows<D>::template store<T>(dk, seen ? a.scale / range : 0.f, a.dk + first, at, S.n - wave * 32, own, lane,
                                 a.dim / 8);
  WaveRows<D>::template store<T>(dv, T::kNarrow ? 1.f / kPScale : 1.f, a.dv + first, at, S.n - wave * 32, own, lane, a.dim / 8);
}

// (The bodies are device functions: the host pass knows no buffer resources.)
template <class T, int D, int NW, int KEYS, int NST, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void attn_fwd_kernel(AttnArgs a) {
  attn_fwd<T, D, NW, KEYS, NST>(a);
}
template <class T, int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_dq_kernel(AttnArgs a) {
  attn_dq<T, D, NW>(a);
}
template <class T, int D, int NW>
__global__ __launch_bounds__(64 * NW, D >= 128 ? 2 : 3) void attn_dkv_kernel(AttnArgs a) {
  attn_dkv<T, D, NW>(a);
}

// The forward's kernels:
//   kFew    a wave, 32 slots, on its own, 32 keys a stage: calls of at most 32 slots a sequence (a
//           token of each of many answers).  No wave idles over slots that are not there and none
//           waits for another; five fit a CU, which keeps the keys' stream going.
//           Its loads pass the caches by: 64 caches of up to 8,192 keys, 222 -> 201 us, and small
//           ones (34 MB) as fast as with them.
//   kShort  4 waves, 128 slots, 32 keys a stage in three stages (64 in two at up to 64 values a head) at
//           three workgroups per CU
//   kLong   4 waves, 128 slots, 64 keys a stage at two workgroups per CU
// kShort against kLong, 32,768 tokens in causal sequences of n, 32 heads of 128, us: n = 128 155 and 178, 512
// 226 and 239, 1,024 352 and 356, 2,048 598 and 597, 4,096 1,104 and 1,058, 8,192 2,108 and 2,029.
enum FwdShape { kFew, kShort, kLong };
constexpr int64_t kLongFrom = 2048;  // mean keys per sequence
FwdShape attn_shape(int64_t n_q, int64_t n_k, int n_seq, int G) {
  if (n_q * G <= 32 * (int64_t)n_seq) return kFew;
  return n_k < kLongFrom * n_seq ? kShort : kLong;
}
int fwd_slots(int64_t n_q, int64_t n_k, int n_seq, int G) {
  return attn_shape(n_q, n_k, n_seq, G) == kFew ? 32 : 128;
}
constexpr int kBwdWaves = 4;
constexpr int kKeyTile = 32 * kBwdWaves;

// Writes the tiles of query rows (numbers below q_tiles), then those of key rows, a wave each: 4 to 5 us,
// mostly its launch.
__global__ __launch_bounds__(256) void plan_kernel(AttnArgs a, uint32_t q_tiles, uint32_t k_tiles, int ts) {
  const uint32_t i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= q_tiles + k_tiles) return;
  const AttnTile t = i < q_tiles ? find_q_tile(a, i, ts) : find_k_tile(a, i - q_tiles, kKeyTile);
  if ((threadIdx.x & 63) == 0) *(i < q_tiles ? a.q_plan + i : a.k_plan + (i - q_tiles)) = t;
}

hipError_t run_plan(const AttnArgs& a, int64_t q_tiles, int64_t k_tiles, int ts, hipStream_t s) {
  if (q_tiles + k_tiles == 0) return hipSuccess;
  hipLaunchKernelGGL(plan_kernel, dim3((unsigned)((q_tiles + k_tiles + 3) / 4)), dim3(256), 0, s, a,
                     (uint32_t)q_tiles, (uint32_t)k_tiles, ts);
  return hipGetLastError();
}

template <class T, int D, int NW, int KEYS, int NST, int OCC>
hipError_t run_fwd_as(const AttnArgs& a, hipStream_t s) {
  const int64_t each = a.tiles * a.splits;
  const int64_t grid = (NW > 1 ? each : (each + 7) / 8 * 8) * a.kv_heads;
  hipError_t e = run_plan(a, a.q_plan ? a.tiles : 0, 0, a.ts, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attn_fwd_kernel<T, D, NW, KEYS, NST, OCC>), dim3((unsigned)grid), dim3(64 * NW), 0,
                     s, a);
  e = hipGetLastError();
  if (e == hipSuccess && a.splits > 1) {
    const int64_t rows = a.n_q * a.heads;
    hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <class T, int D>
hipError_t run_fwd(const AttnArgs& a, hipStream_t s) {
  switch (attn_shape(a.n_q, a.n_k, a.n_seq, a.G)) {
    case kFew: return run_fwd_as<T, D, 1, 32, 2, 2>(a, s);
    case kShort: return run_fwd_as<T, D, 4, D >= 128 ? 32 : 64, D >= 128 ? 3 : 2, 3>(a, s);
    default: return run_fwd_as<T, D, 4, 64, 2, 2>(a, s);
  }
}

template <class T, int D>
hipError_t run_bwd(AttnArgs a, hipStream_t s) {
  const int ts = 32 * kBwdWaves / a.G;
  const int64_t q_tiles = a.n_q > 0 ? a.n_q / ts + a.n_seq : 0;
  const int64_t k_tiles = a.dk && a.n_k > 0 ? a.n_k / kKeyTile + a.n_seq : 0;
  hipError_t e = run_plan(a, a.q_plan ? q_tiles : 0, a.k_plan ? k_tiles : 0, ts, s);
  if (e == hipSuccess && q_tiles > 0) {
    a.ts = ts;
    a.tiles = q_tiles;
    hipLaunchKernelGGL((attn_dq_kernel<T, D, kBwdWaves>), dim3((unsigned)(q_tiles * a.kv_heads)),
                       dim3(64 * kBwdWaves), 0, s, a);
    e = hipGetLastError();
  }
  if (e == hipSuccess && k_tiles > 0) {
    a.ts = kSlots / a.G;
    a.tiles = k_tiles;
    hipLaunchKernelGGL((attn_dkv_kernel<T, D, kBwdWaves>), dim3((unsigned)(k_tiles * a.kv_heads)),
                       dim3(64 * kBwdWaves), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// Splits of the key axis, where the tiles alone do not fill the chip: none of fewer than 128 keys of the
// mean sequence.
//   kFew, from 512 keys: four waves per CU, or up to sixteen of no fewer than 512 keys, which evens out
//     sequences of different lengths.  A token each, 8 kv heads of 128, us (equal sequences of 4,096 keys;
//     uneven ones of 64 to 8,192): 8 sequences in 16 splits 29; 42, in 32 33; 50.  32 in 4 splits 91; 102, in
//     8 92; 89, in 16 101; 93.  64 in 2 splits 178; 220, in 8 181; 191, in 16 195; 195.  16 of 700 keys 22
//     whole, 15 in 5.
//   Others: a split's sums go out and come back as fp32, so the split of the least estimated time, from what
//     workgroups take on their own (18 ns a key, 14 at 64 values a head), half as long again when most CUs
//     hold two, the join's launch (4 us) and 4 TB/s for its sums.  32 heads of 128, 8 kv heads: 128 rows of 2
//     sequences of 4,096 keys 77 -> 37 us, of 8 sequences 107 -> 86, 512 rows of one 75 -> 49; left whole: a
//     sequence of 512 rows 21 us (two splits 23), 4 sequences of 512 with 12 heads of 64 11 us (24).
int attn_splits(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, int dim) {
  constexpr int kCus = 256;
  if (n_q < 1) return 1;
  const int G = heads / kv_heads;
  const bool few = attn_shape(n_q, n_k, n_seq, G) == kFew;
  const int64_t ts = fwd_slots(n_q, n_k, n_seq, G) / G, mean = n_k / n_seq;
  // workgroups that hold tokens, if the sequences are of one length
  const int64_t live = n_q < n_seq ? n_q : n_seq;
  const int64_t wgs = live * ((n_q / live + ts - 1) / ts) * kv_heads;
  if (wgs >= (few ? 16 : 2) * kCus) return 1;
  int64_t most = mean / 128 < kMaxSplits ? mean / 128 : kMaxSplits;
  // (the grid also has the tiles of empty sequences: no more than 2^22 workgroups for the splits' sake)
  const int64_t grid = (n_q / ts + n_seq) * kv_heads;
  if (most > (int64_t(1) << 22) / grid) most = (int64_t(1) << 22) / grid;
  if (few) {
    if (mean < 512 || most < 1) return 1;
    const int64_t four = (4 * kCus + wgs - 1) / wgs, all = (16 * kCus + wgs - 1) / wgs, wide = mean / 512;
    const int64_t s = all < wide ? all : wide;
    return (int)((s > four ? s : four) < most ? (s > four ? s : four) : most);
  }
  const double sums = (double)n_q * heads * dim * 8 / 4e6;  // us a split, out and back
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= most; ++s) {
    const int64_t w = wgs * s;
    const double share = w <= 3 * kCus / 4 ? 1. : w <= 2 * kCus ? 1.5 : 1.6 * w / (2 * kCus);
    const double us = (double)mean / s * (dim > 64 ? 0.018 : 0.014) * share + (s > 1 ? 4. + s * sums : 0.);
    if (us < least) least = us, best = s;
  }
  return best;
}

// Calls of at least four rounds of workgroups plan their tiles.  n sequences of 250 tokens, 32 heads of 128 on
// 8 kv heads, us planned (searched by every workgroup): forward n = 32 (2,256 tiles) 44 (43), 64 86 (85), 128
// 158 (163), 256 304 (320), 1,024 of 60 tokens 223 (238); gradients 132 (133), 250 (252), 483 (488), 937
// (961), 682 (714).
constexpr int64_t kPlanFrom = 2048;

int64_t attn_plan_tiles(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads) {
  if (n_q < 1) return 0;
  const int G = heads / kv_heads;
  const int64_t tiles = n_q / (fwd_slots(n_q, n_k, n_seq, G) / G) + n_seq;
  return tiles * kv_heads >= kPlanFrom ? tiles : 0;
}

int64_t attn_plan_q_tiles(int64_t n_q, int n_seq, int heads, int kv_heads) {
  if (n_q < 1) return 0;
  const int64_t tiles = n_q / (32 * kBwdWaves / (heads / kv_heads)) + n_seq;
  return tiles * kv_heads >= kPlanFrom ? tiles : 0;
}

int64_t attn_plan_key_tiles(int64_t n_k, int n_seq, int kv_heads) {
  if (n_k < 1) return 0;
  const int64_t tiles = n_k / kKeyTile + n_seq;
  return tiles * kv_heads >= kPlanFrom ? tiles : 0;
}

// (Split calls are of at most 2^22 workgroups, and the plans' and the join's launches smaller than these.)
bool attn_fits(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, bool grads) {
  const int G = heads / kv_heads;
  if (!grads) {
    if (n_q == 0) return true;
    const bool few = attn_shape(n_q, n_k, n_seq, G) == kFew;
    const int64_t tiles = n_q / (fwd_slots(n_q, n_k, n_seq, G) / G) + n_seq;
    return launch_fits((tiles + (few ? 7 : 0)) * kv_heads, few ? 64 : 256);
  }
  const int64_t q_tiles = n_q / (32 * kBwdWaves / G) + n_seq, k_tiles = n_k / kKeyTile + n_seq;
  return launch_fits((q_tiles > k_tiles ? q_tiles : k_tiles) * kv_heads, 64 * kBwdWaves);
}

hipError_t launch_attn_fwd(AttnArgs a, hipStream_t stream) {
  if (a.n_q == 0) return hipSuccess;
  a.ts = fwd_slots(a.n_q, a.n_k, a.n_seq, a.G) / a.G;
  a.tiles = a.n_q / a.ts + a.n_seq;
  if (a.f16) return a.dim <= 64 ? run_fwd<HalfF16, 64>(a, stream) : run_fwd<HalfF16, 128>(a, stream);
  return a.dim <= 64 ? run_fwd<HalfBf16, 64>(a, stream) : run_fwd<HalfBf16, 128>(a, stream);
}

hipError_t launch_attn_bwd(AttnArgs a, hipStream_t stream) {
  if (a.f16) return a.dim <= 64 ? run_bwd<HalfF16, 64>(a, stream) : run_bwd<HalfF16, 128>(a, stream);
  return a.dim <= 64 ? run_bwd<HalfBf16, 64>(a, stream) : run_bwd<HalfBf16, 128>(a, stream);
}

}  // namespace hpr
