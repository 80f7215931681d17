// Shared pieces of the training attention kernels (train_fwd.hip, train_dq.hip,
// train_dkv.hip): records the host hands them, LDS tile layout, fragment reads
// and products, for bf16 and fp32 tensors of packed rows.
//
// Mathematics. For query row i and key row j of one group (a history, or a
// user's events and history)
//   t_ij = scale q_i.k_j + bias(i, j),  P = softmax over the visible j,
//   O_i = sum_j P_ij v_j,  lse_i = log sum_j exp(t_ij)
// and, given dO,
//   D_i = dO_i.O_i,  dS_ij = P_ij (dO_i.v_j - D_i),
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,
//   dv_j = sum_i P_ij dO_i,  dbias_b = sum over pairs of bucket b of dS_ij.
// P is recomputed from lse, so nothing of the size of t is kept. Logits live in
// the base-2 domain (scaled by log2 e, exponentiated with exp2), fp32.
#pragma once

#include "tx_internal.h"
#include "wave_reduce.h"

#include <mutex>

namespace tx {

// A group of a call, rows counted from the start of the tensors. Units are the
// blocks of work of a launch per head: for query-side launches (forward, dq)
// the group owns units unit_q .. , parts_q per block of queries, for the
// key-side launch (dk, dv) unit_k .. , parts_k per block of keys. Groups whose
// blocks are divided (parts > 1) keep their partial results in slots from slot_q / slot_k on, which a second launch joins in the order of
// the parts (joining them in the block that finishes last saves that launch,
// but the fences write whole L2 caches back: one token against 4096 keys took
// 131 us so, of 64 parts a head). qt0: its first entry in the 64-row query
// tile list; e0 .. e1 - 1: its events.
struct TrainGroup {
  int32_t q0, nq, k0, nk;
  int32_t unit_q, parts_q, slot_q, qt0;
  int32_t unit_k, parts_k, slot_k, e0;
  int32_t e1, pad[3];
};
// Rows of a block: queries (forward, dq) or keys (dk, dv). Wide blocks give each of
// their four waves 32 of 128 rows and share the tiles of the other side. Narrow
// ones give all four the same 32 rows and every fourth tile, each wave with
// buffers of its own and no barrier between tiles, and add up at the end: for
// calls whose wide blocks would leave most of the card idle, each with a long
// chain of tiles. Where query heads share a key head (and no bias tells them
// apart), a wide block of queries packs 2 or 4 of them: its waves take the same
// 64 or 32 rows of several heads, so that few rows still fill it and read the
// keys and values once.
constexpr int kWideRows = 128, kNarrowRows = 32;
constexpr int kTrainQTile = 64;   // granularity of the per-tile key limits
constexpr int kTrainMaxRel = 2048;

struct TileLim {
  int32_t lo, hi;  // smallest and largest number of visible keys among a tile's rows
};

// Rows of a tensor: element (row, head, f) at p + row * row + head * head
// bytes + f elements.
struct HeadRows {
  char* p;
  int64_t row, head;
};

struct TrainArgs {
  const TrainGroup* groups;
  int32_t n_groups, H, G;  // H query heads, G key heads
  int32_t n_units, q_chunk, k_units, k_chunk;  // units of either side and their place_chunk
  const uint32_t *q_order, *k_order;  // units by work, group + 65536 local; null: group after group
  HeadRows q, k, v, o, dO, dq, dk, dv;
  float* lse;           // [H][lse_ld], natural logarithm
  int64_t lse_ld;
  float* row_stat;      // [H][stat_ld][2]: lse in base 2 (infinite for a row that sees nothing) and D, from
                        // row q_base on; dq writes them, dk and dv read them
  int64_t stat_ld;
  const void* rel;      // [H][R] in the tensors' type
  int32_t R;
  const int32_t* row_lim;   // event form: visible keys of each query row (from row q_base on; room for an even number)
  const TileLim* tile_lim;
  int32_t q_base;
  float scale, scale_log2;
  float* partial;       // slots of divided blocks
  int32_t q_rows, k_rows;   // rows of a query-side and of a key-side block
  bool q_narrow, k_narrow;
  int32_t pack;             // log2 of the query heads in a wide query-side block
  float* drel_part;     // [unit][H][R] sums of dS by bucket
};

hipError_t launch_train_fwd(bool bf, int dh, bool rel, const TrainArgs& a, hipStream_t s);
hipError_t launch_train_fwd_join(bool bf, int dh, const TrainArgs& a, hipStream_t s);
hipError_t launch_train_dq(bool bf, int dh, bool rel, const TrainArgs& a, hipStream_t s);
hipError_t launch_train_dq_join(bool bf, int dh, const TrainArgs& a, hipStream_t s);
hipError_t launch_train_dkv(bool bf, int dh, bool rel, const TrainArgs& a, hipStream_t s);
hipError_t launch_train_dkv_join(bool bf, int dh, const TrainArgs& a, hipStream_t s);
// drel[h][b] from the units' sums; scratch: [chunks][H][R] floats, chunks = ceil(units / 32)
hipError_t launch_train_drel(bool bf, const TrainArgs& a, float* scratch, void* drel, hipStream_t s);
// row_lim and tile_lim of the event form (n_tiles > 0) from the groups and the
// events' row offsets and prefixes: from memory, or from metadata of at most
// sizeof(MetaArg) bytes (groups first) that is written to dst by the way
hipError_t launch_train_limits(const TrainGroup* groups, int32_t n_groups, int32_t n_tiles, const int32_t* ev_row,
                               const int32_t* ev_prefix, int32_t* row_lim, int32_t q_base, TileLim* tile_lim,
                               hipStream_t s);
hipError_t launch_train_put_limits(void* dst, const void* meta, size_t bytes, int32_t n_groups, int32_t n_tiles,
                                   size_t o_row, size_t o_prefix, int32_t* row_lim, int32_t q_base, TileLim* tile_lim,
                                   hipStream_t s);

// Blocks go to the card's 8 XCDs in turn, each with an L2 of its own, and the
// units of a group read the same rows of the other side. With a multiple of 8
// heads (or packed heads) a launch runs over the heads first, so that a head
// stays on one XCD. With 1, 2 or 4 an XCD gets one head and up to 32 units in a
// row of it, then skips what the XCDs of the same head take: dk and dv of 147 k
// queries of 2.3 k keys, 8 heads on 2 key heads: 4.48 -> 3.50 ms. Other counts run over the
// heads first as well.
__host__ __device__ inline bool placed(int heads) { return heads == 1 || heads == 2 || heads == 4; }
inline int place_chunk(int64_t units, int heads) {
  if (!placed(heads) || units == 0) return 0;
  const int64_t xcds = 8 / heads, rounds = (units + 32 * xcds - 1) / (32 * xcds);
  return (int)((units + xcds * rounds - 1) / (xcds * rounds));
}
inline unsigned place_grid(int64_t units, int heads, int chunk) {
  if (!chunk) return (unsigned)(units * heads);
  const int64_t round = (int64_t)chunk * (8 / heads);
  return (unsigned)((units + round - 1) / round * round * heads);
}

// floats of one partial slot
__host__ __device__ inline size_t train_fwd_slot(int rows, int dh) { return (size_t)rows * (dh + 2); }
__host__ __device__ inline size_t train_dq_slot(int rows, int dh) { return (size_t)rows * dh; }
__host__ __device__ inline size_t train_dkv_slot(int rows, int dh) { return (size_t)2 * rows * dh; }

// LDS of a block of the dq kernel: its tiles and the bias tables of R buckets;
// what a CU has for one block, less the compiler's own.
size_t train_dq_lds(bool bf, int dh, int R, bool narrow);
constexpr size_t kTrainMaxLds = 159 * 1024;

#ifdef __HIPCC__

constexpr float kTrainLog2e = 1.4426950408889634f, kTrainLn2 = 0.6931471805599453f;
constexpr float kBiasMasks = -1e30f;  // a bias at or below it masks (the lowest values of bf16 and fp32 do)
// Entries of the padded bias table on either side of the buckets: distances
// from -kBiasPad (not visible) to R - 1 + kBiasPad (last bucket) of a tile that
// touches the buckets.
constexpr int kBiasPad = 96;
__host__ __device__ inline int bias_entries(int R) { return R + 2 * kBiasPad; }

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
typedef __attribute__((address_space(3))) u32x2_t lds_u32x2;
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) floatx4 lds_floatx4;
typedef __attribute__((address_space(3))) int lds_int;

// The group of unit u: the last one whose first unit is <= u (64-ary search by
// the lanes of a wave; uniform).
template <bool KEY_SIDE>
__device__ __forceinline__ int find_group(const TrainGroup* __restrict__ g, int n, int u, int lane) {
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    bool ok = false;
    if (i < n) ok = (KEY_SIDE ? g[lo + i].unit_k : g[lo + i].unit_q) <= u;
    const int c = max(1, (int)__popcll(__ballot(ok)));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Geometry of a tile of rows of DH elements in LDS. 16-byte unit u of row r
// sits at u ^ swz(r). swz is linear over the bits of r, is different for 16
// neighbouring rows (row-wise fragment reads: 16 lanes per pass read the same
// unit of 16 rows) and moves 4 neighbouring rows to different groups of 4
// units (the transposing reads of bf16 tiles take 4 units of 4 rows at a time),
// so both reads spread over the 64 banks.
template <class T, int DH>
struct Geo {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int RB = DH * (int)sizeof(T);  // bytes of a row
  static constexpr int UPR = RB / 16;
  static constexpr int NC = RB / 32;              // 32-byte chunks: two lanes' fragments each
  static constexpr int NB = DH / 32;              // 32-feature blocks of an accumulator
  static __host__ __device__ constexpr int swz(int r) {
    return BF ? (UPR == 16  ? ((r & 3) << 2) | ((r >> 2) & 3)
                 : UPR == 8 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3)
                            : (r >> 2) & 3)
              : (UPR >= 16 ? ((r & 4) << 1) | ((r & 8) >> 1) | (r & 3) : (r >> 1) & 7);
  }
};

// Fragment reads and products of one wave.
//   row fragment c of row r: the lane's 16 bytes (lanes 0-31 the first half of
//   chunk c of rows 0 .. 31, lanes 32-63 the second half)
//   rows_mma: acc[m][n] += sum_f A[m][f] B[n][f] from row fragments
//   cols_mma: acc[f][n] += sum_r tile[r][f] X[r][n], X in the accumulator
//   layout (lane: column n = lane % 32, register v: row 8 (v / 4) + 4 (lane /
//   32) + v % 4), which is the layout in which X was computed
//
// Scheduling: N fragment reads (R LDS reads each) for N products of M matrix
// instructions, the reads AHEAD fragments in front; left to itself the
// compiler hoists all the reads and spills.
template <int N, int R, int M, int AHEAD = 4>
__device__ __forceinline__ void pace() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * R, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD * M, 0);
}

template <class T, int DH>
struct Wave {
  using G = Geo<T, DH>;
  static constexpr bool BF = G::BF;
  int row_off, col_off;  // lane parts of the LDS byte offsets
  __device__ __forceinline__ explicit Wave(int lane) {
    const int l32 = lane & 31, hi = lane >> 5;
    row_off = l32 * G::RB + ((hi ^ G::swz(l32)) << 4);
    if (BF) {
      const int i = lane & 15, half = (lane >> 4) & 1, r = 4 * hi + (i >> 2);
      col_off = r * G::RB + (((2 * half + ((i & 3) >> 1)) ^ G::swz(r)) << 4) + ((i & 1) << 3);
    } else {
      col_off = 4 * hi * G::RB + (((l32 >> 2) ^ G::swz(4 * hi)) << 4) + ((l32 & 3) << 2);
    }
  }
  // Tiles start at multiples of 1024 bytes, so the swizzle's XOR, which stays
  // within a row, can follow the addition of the tile's address: one addition
  // for all fragments of a tile.
  static __device__ __forceinline__ uint32_t lds_address(const lds_char* p) { return (uint32_t)(uintptr_t)p; }
  __device__ __forceinline__ u32x4_t row_frag(const lds_char* tile, int rb, int c) const {
    const uint32_t at = (lds_address(tile) + row_off) ^ (c << 5);
    return *((const lds_u32x4*)(uintptr_t)at + rb * 2 * G::RB);
  }
  static __device__ __forceinline__ floatx16 rows_mma(u32x4_t a, u32x4_t b, floatx16 c) {
    if constexpr (BF) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                     0, 0);
    } else {
      const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
      for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[t], y[t], c, 0, 0, 0);
      return c;
    }
  }
  // bf16: 8 rows of column 32 db + lane % 32, rows 32 rb + 16 h + 8 (t / 4) + 4 (lane / 32) + t % 4
  __device__ __forceinline__ bf16x8 col_frag(const lds_char* tile, int rb, int h, int db) const {
    const uint32_t at = lds_address(tile) + col_off;
    lds_s16x4* const pa = (lds_s16x4*)(uintptr_t)(at ^ (db << 6)) + (32 * rb + 16 * h) * (G::RB / 8);
    lds_s16x4* const pb =
        (lds_s16x4*)(uintptr_t)(at ^ ((db << 6) | (G::swz(8) << 4))) + (32 * rb + 16 * h + 8) * (G::RB / 8);
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(pa);
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(pb);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // fp32: row 32 rb + 8 (v / 4) + 4 (lane / 32) + v % 4 of column 32 db + lane % 32
  __device__ __forceinline__ float col_elem(const lds_char* tile, int rb, int v, int db) const {
    const int rc = 8 * (v >> 2) + (v & 3);
    return *reinterpret_cast<const lds_float*>(tile + (32 * rb + rc) * G::RB +
                                               (col_off ^ (((8 * db) ^ G::swz(rc)) << 4)));
  }
  static __device__ __forceinline__ bf16x8 pack(const floatx16& x, int h) {
    bf16x8 p;
#pragma unroll
    for (int t = 0; t < 8; ++t) p[t] = (bf16)x[8 * h + t];
    return p;
  }
  __device__ __forceinline__ void cols_mma(const lds_char* tile, int rb, const floatx16& x,
                                           floatx16 (&acc)[G::NB]) const {
    if constexpr (BF) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 p = pack(x, h);
#pragma unroll
        for (int db = 0; db < G::NB; ++db)
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(col_frag(tile, rb, h, db), p, acc[db], 0, 0, 0);
      }
      if constexpr (G::NB >= 2) pace<2 * G::NB, 2, 1>();
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int db = 0; db < G::NB; ++db)
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(col_elem(tile, rb, v, db), x[v], acc[db], 0, 0, 0);
    }
  }
  // a = A B^T of the 32 rows rb of a tile, and the same of a second tile
  __device__ __forceinline__ void rows_product(const lds_char* tile, int rb, const u32x4_t (&f)[G::NC],
                                               floatx16& a) const {
#pragma unroll
    for (int v = 0; v < 16; ++v) a[v] = 0.f;
#pragma unroll
    for (int c = 0; c < G::NC; ++c) a = rows_mma(row_frag(tile, rb, c), f[c], a);
    if constexpr (BF && G::NC >= 4) pace<G::NC, 1, 1>();
  }
  // (the second added to what a2 holds)
  template <int FIRST = 0>
  __device__ __forceinline__ void rows_products(const lds_char* t1, const u32x4_t (&f1)[G::NC], floatx16& a1,
                                                const lds_char* t2, const u32x4_t (&f2)[G::NC], floatx16& a2,
                                                int rb) const {
#pragma unroll
    for (int v = 0; v < 16; ++v) a1[v] = 0.f;
    if constexpr (BF && FIRST > 0) __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
#pragma unroll
    for (int c = 0; c < G::NC; ++c) {
      a1 = rows_mma(row_frag(t1, rb, c), f1[c], a1);
      a2 = rows_mma(row_frag(t2, rb, c), f2[c], a2);
    }
    if constexpr (BF) pace<2 * G::NC, 1, 1>();
  }
  // rows_products with the second operand's fragments of the second product in
  // LDS too (32 rows at t3)
  __device__ __forceinline__ void rows_products_lds(const lds_char* t1, const u32x4_t (&f1)[G::NC], floatx16& a1,
                                                    const lds_char* t2, const lds_char* t3, floatx16& a2,
                                                    int rb) const {
#pragma unroll
    for (int v = 0; v < 16; ++v) a1[v] = 0.f;
    if constexpr (BF) __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int c = 0; c < G::NC; ++c) {
      a1 = rows_mma(row_frag(t1, rb, c), f1[c], a1);
      a2 = rows_mma(row_frag(t2, rb, c), row_frag(t3, 0, c), a2);
    }
    if constexpr (BF) {
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
      for (int i = 0; i < G::NC - 2; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }
  }
  // cols_mma of two tiles
  __device__ __forceinline__ void cols_mma2(const lds_char* t1, const floatx16& x1, floatx16 (&acc1)[G::NB],
                                            const lds_char* t2, const floatx16& x2, floatx16 (&acc2)[G::NB],
                                            int rb) const {
    if constexpr (BF) {
      const bf16x8 p[2] = {pack(x1, 0), pack(x1, 1)}, r[2] = {pack(x2, 0), pack(x2, 1)};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int db = 0; db < G::NB; ++db) {
          acc1[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(col_frag(t1, rb, h, db), p[h], acc1[db], 0, 0, 0);
          acc2[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(col_frag(t2, rb, h, db), r[h], acc2[db], 0, 0, 0);
        }
      pace<4 * G::NB, 2, 1>();
    } else {
      cols_mma(t1, rb, x1, acc1);
      cols_mma(t2, rb, x2, acc2);
    }
  }
  // Whether the 32 rows hold an infinity or a NaN (uniform).
  __device__ __forceinline__ bool rows_not_finite(const lds_char* tile, int rb) const {
    uint32_t bad = 0;
#pragma unroll
    for (int c = 0; c < G::NC; ++c) {
      const u32x4_t w = row_frag(tile, rb, c);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        bad |= BF ? ((w[t] & 0x7f807f80u) + 0x00800080u) & 0x80008000u
                  : ((w[t] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
    }
    return __any(bad != 0);
  }
  // cols_mma for rows that hold infinities or NaN and an X whose bit v of
  // `vis` tells whether X's register v belongs to a visible pair: a masked pair
  // adds nothing (0 x NaN would), a visible one makes the sum NaN. The finite
  // values go through the same product in the same order, and a second product
  // of indicators finds the sums that a value not finite reaches, so the other
  // sums keep their bits. Rare.
  __device__ __forceinline__ void cols_mma_strict(const lds_char* tile, int rb, const floatx16& x, uint32_t vis,
                                                  floatx16 (&acc)[G::NB]) const {
#pragma unroll
    for (int db = 0; db < G::NB; ++db) {
      floatx16 hit;
#pragma unroll
      for (int v = 0; v < 16; ++v) hit[v] = 0.f;
      if constexpr (BF) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 a = col_frag(tile, rb, h, db), bad, seen;
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const bool fin = __builtin_isfinite((float)a[t]);
            bad[t] = fin ? (bf16)0.f : (bf16)1.f;
            a[t] = fin ? a[t] : (bf16)0.f;
            seen[t] = (vis >> (8 * h + t)) & 1 ? (bf16)1.f : (bf16)0.f;
          }
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pack(x, h), acc[db], 0, 0, 0);
          hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bad, seen, hit, 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if (v % 4 == 0) __builtin_amdgcn_sched_barrier(0);
          const float a = col_elem(tile, rb, v, db);
          const bool fin = __builtin_isfinite(a);
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(fin ? a : 0.f, x[v], acc[db], 0, 0, 0);
          hit = __builtin_amdgcn_mfma_f32_32x32x2f32(fin ? 0.f : 1.f, (vis >> v) & 1 ? 1.f : 0.f, hit, 0, 0, 0);
        }
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] = hit[v] > 0.f ? __builtin_nanf("") : acc[db][v];
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Copies of ROWS rows of DH elements from a tensor into an LDS tile, straight
// from HBM/L2 (no registers), by the four waves of a block: piece p (1 KB of
// the tile) goes to wave p % 4. Rows past `rows` read as zeros (they lie beyond
// the buffer resource's extent). The swizzle is applied on the global side.
//
// The loads are written in asm (they have no result registers; the LDS address
// of the wave's 1 KB is in m0): behind the builtin the compiler makes every
// transposing LDS read wait for all loads in flight, the next tile's among
// them. So nothing waits for them but tiles_ready().
// HELD: the lane's offsets stay in registers; otherwise they are made anew for
// every tile. WAVES = 1: the wave copies the tile alone (wave index 0).
template <class T, int DH, int ROWS, bool HELD = true, int WAVES = 4>
struct TileDma {
  using G = Geo<T, DH>;
  static constexpr int PER = ROWS * G::RB / (1024 * WAVES);  // pieces of a wave
  uint32_t off[HELD ? PER : 1];
  int wave, lane;
  uint32_t ldb;
  __device__ __forceinline__ uint32_t offset(int u, int l) const {
    const int r = (wave + WAVES * u) * (1024 / G::RB) + l / G::UPR, s = l % G::UPR;
    return (uint32_t)r * ldb + ((uint32_t)(s ^ G::swz(r)) << 4);
  }
  __device__ __forceinline__ TileDma(int wave_, int lane_, int64_t row_bytes)
      : wave(wave_), lane(lane_), ldb((uint32_t)row_bytes) {
    if (HELD)
#pragma unroll
      for (int u = 0; u < PER; ++u) off[u] = offset(u, lane);
  }
  // rows: rows left in the tensor's group from `first` on (>= 1)
  __device__ __forceinline__ void load(const char* first, int rows, lds_char* tile) const {
    const int n = min(rows, ROWS);
    const uint64_t at = (uint64_t)first;
    // (uniform() where the compiler does not see it)
    const u32x4_t r = {(uint32_t)uniform((int)at), (uint32_t)uniform((int)(at >> 32)) & 0xffffu,
                       (uint32_t)uniform((n - 1) * (int)ldb) + G::RB, 0x00020000u};
    const uint32_t to = uniform((int)(uint32_t)(uintptr_t)tile) + wave * 1024;
    int l = lane;
    if (!HELD) asm volatile("" : "+v"(l));  // not hoisted
#pragma unroll
    for (int u = 0; u < PER; ++u)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :
                   : "s"(to + u * 1024 * WAVES), "v"(HELD ? off[HELD ? u : 0] : offset(u, l)), "s"(r)
                   : "m0", "memory");
  }
};

// Every wave's copies into LDS have landed and every wave is past its last reads.
__device__ __forceinline__ void tiles_ready() {
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  asm volatile("" ::: "memory");
  __syncthreads();
}

// The lane's fragments of one row (lane % 32) straight from memory; zeros
// where the row does not exist.
template <class T, int DH>
__device__ __forceinline__ void load_row_frags(const char* row, bool exists, int hi, u32x4_t (&f)[Geo<T, DH>::NC]) {
#pragma unroll
  for (int c = 0; c < Geo<T, DH>::NC; ++c) f[c] = u32x4_t{0, 0, 0, 0};
  if (exists) {
#pragma unroll
    for (int c = 0; c < Geo<T, DH>::NC; ++c) f[c] = *reinterpret_cast<const u32x4_t*>(row + 32 * c + 16 * hi);
  }
}

// For a wave on its own: its copies have landed, and its reads of the tile before
// are done, so that the next copies may go there (LDS reads and copies into LDS
// are not ordered by themselves).
__device__ __forceinline__ void tile_ready() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
}
// Its reads alone.
__device__ __forceinline__ void tile_read() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// Waits for values loaded from memory: left to the compiler, the wait would sit
// at their first use, inside a loop over tiles, where it would also wait for the
// tiles in flight.
template <int N>
__device__ __forceinline__ void pin(u32x4_t (&f)[N]) {
#pragma unroll
  for (int c = 0; c < N; ++c) asm volatile("" : "+v"(f[c]));
}
template <class T>
__device__ __forceinline__ void pin(T& x) {
  asm volatile("" : "+v"(x));
}

// Parks a wave's accumulator (columns = rows of the output, 32 of them) in LDS
// as output rows in T and stores them row-contiguously, 16 bytes a lane. stage:
// 32 * RB bytes of this wave's own. mul: factor of the lane's column.
template <class T, int DH>
__device__ __forceinline__ void store_rows(const floatx16 (&acc)[Geo<T, DH>::NB], float mul, lds_char* stage, char* out,
                                           int64_t row_bytes, int n_rows, int lane) {
  using G = Geo<T, DH>;
  const int l32 = lane & 31, hi = lane >> 5;
#pragma unroll
  for (int db = 0; db < G::NB; ++db)
#pragma unroll
    for (int gq = 0; gq < 4; ++gq) {
      if constexpr (G::BF) {
        bf16x4 w;
#pragma unroll
        for (int t = 0; t < 4; ++t) w[t] = (bf16)(acc[db][4 * gq + t] * mul);
        *reinterpret_cast<lds_u32x2*>(stage + l32 * G::RB + (((4 * db + gq) ^ G::swz(l32)) << 4) + 8 * hi) =
            __builtin_bit_cast(u32x2_t, w);
      } else {
        floatx4 w;
#pragma unroll
        for (int t = 0; t < 4; ++t) w[t] = acc[db][4 * gq + t] * mul;
        *reinterpret_cast<lds_u32x4*>(stage + l32 * G::RB + (((8 * db + 2 * gq + hi) ^ G::swz(l32)) << 4)) =
            __builtin_bit_cast(u32x4_t, w);
      }
    }
  __builtin_amdgcn_wave_barrier();
  constexpr int RPI = 64 / G::UPR;
#pragma unroll
  for (int k = 0; k < 32 / RPI; ++k) {
    const int r = k * RPI + lane / G::UPR, u = lane % G::UPR;
    const u32x4_t w = *reinterpret_cast<const lds_u32x4*>(stage + r * G::RB + ((u ^ G::swz(r)) << 4));
    if (r < n_rows) *reinterpret_cast<u32x4_t*>(out + r * row_bytes + 16 * u) = w;
  }
}

// The accumulator as fp32 rows of a partial slot (row = the lane's column).
template <class T, int DH>
__device__ __forceinline__ void store_partial(const floatx16 (&acc)[Geo<T, DH>::NB], float* row, int hi) {
#pragma unroll
  for (int db = 0; db < DH / 32; ++db)
#pragma unroll
    for (int gq = 0; gq < 4; ++gq) {
      floatx4 w;
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = acc[db][4 * gq + t];
      *reinterpret_cast<floatx4*>(row + 32 * db + 8 * gq + 4 * hi) = w;
    }
}

// Four floats of an output row.
template <class T>
__device__ __forceinline__ void store4(T* to, floatx4 x, float mul) {
  if constexpr (sizeof(T) == 2) {
    bf16x4 y;
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] = (bf16)(x[t] * mul);
    *reinterpret_cast<bf16x4*>(to) = y;
  } else {
    floatx4 y;
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] = x[t] * mul;
    *reinterpret_cast<floatx4*>(to) = y;
  }
}

// How a block of 256 threads goes through `rows` partial rows of DH floats: DH /
// 4 threads a row, as many rows at once as there are threads or rows, and what
// threads are left over on shares of the parts.
template <int DH>
struct Joiner {
  static constexpr int LPR = DH / 4, GROUPS = 256 / LPR;
  int f, slot, share, at_once, shares;
  __device__ __forceinline__ Joiner(int rows, int tid) {
    at_once = 1;
    while (at_once < rows && at_once < GROUPS) at_once <<= 1;
    shares = GROUPS / at_once;
    f = tid % LPR * 4;
    slot = tid / LPR % at_once;
    share = tid / LPR / at_once;
  }
};

// out[r] = mul * sum over the parts of rows r of their slots (step floats apart).
template <class T, int DH>
__device__ __forceinline__ void join_sums(const float* p0, size_t step, int parts, int rows, float mul, char* out,
                                          int64_t row_bytes, lds_char* smem, int tid) {
  const Joiner<DH> j(rows, tid);
  lds_floatx4* const left = (lds_floatx4*)smem;
  for (int r0 = 0; r0 < rows; r0 += j.at_once) {
    const int r = r0 + j.slot;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    if (r < rows) {
#pragma unroll 4
      for (int p = j.share; p < parts; p += j.shares) {
        const floatx4 x = *reinterpret_cast<const floatx4*>(p0 + p * step + (size_t)r * DH + j.f);
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] += x[t];
      }
    }
    if (j.shares > 1) {
      left[tid] = acc;
      __syncthreads();
      for (int q = 1; q < j.shares && j.share == 0; ++q) {
        const floatx4 x = left[tid + q * j.at_once * Joiner<DH>::LPR];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] += x[t];
      }
      __syncthreads();
    }
    if (r < rows && j.share == 0) store4((T*)(out + r * row_bytes) + j.f, acc, mul);
  }
}

// Narrow blocks: a wave parks its accumulator (columns = 32 rows of the output)
// as fp32 rows in LDS, 16-byte unit u of row r at u ^ r within units of 8 or 16.
template <int DH>
struct Park {
  static constexpr int UNITS = DH / 4, MASK = UNITS >= 16 ? 15 : 7;
  static constexpr int BYTES = 32 * DH * 4;
  static __device__ __forceinline__ lds_floatx4* at(lds_char* to, int r, int u) {
    return (lds_floatx4*)(to + (r * UNITS + (u ^ (r & MASK))) * 16);
  }
  template <int NB>
  static __device__ __forceinline__ void put(const floatx16 (&acc)[NB], lds_char* to, int lane) {
    const int l32 = lane & 31, hi = lane >> 5;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        floatx4 x;
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = acc[db][4 * gq + t];
        *at(to, l32, 8 * db + 2 * gq + hi) = x;
      }
  }
};
// The sum of the four waves' parked accumulators, row by row: into the output
// (slot null) or a partial slot. `step` bytes between the waves' areas.
template <class T, int DH>
__device__ __forceinline__ void add_parked(lds_char* area, int step, float* slot, float mul, char* out,
                                           int64_t row_bytes, int rows, int tid) {
  using P = Park<DH>;
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) {
    const int r = (tid + 256 * i) / P::UNITS, u = (tid + 256 * i) % P::UNITS;
    floatx4 x = *P::at(area, r, u);
#pragma unroll
    for (int wv = 1; wv < 4; ++wv) {
      const floatx4 y = *P::at(area + wv * step, r, u);
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] += y[t];
    }
    if (r >= rows) continue;
    if (slot) *reinterpret_cast<floatx4*>(slot + r * DH + 4 * u) = x;
    else store4((T*)(out + r * row_bytes) + 4 * u, x, mul);
  }
}

// The head's bias in base-2 units, padded: entry kBiasPad + d is the bias of
// distance d, minus infinity for d < 0. R = 0: no bias.
template <class T>
__device__ __forceinline__ float bias_value(const T* __restrict__ rel, int R, int h, int d) {
  if (d < 0) return -INFINITY;
  if (R == 0) return 0.f;
  const float b = (float)rel[(size_t)h * R + min(d, R - 1)];
  return b <= kBiasMasks ? -INFINITY : b * kTrainLog2e;
}
template <class T>
__device__ __forceinline__ void stage_bias(lds_float* tab, const T* __restrict__ rel, int R, int h, int tid) {
  for (int i = tid; i < bias_entries(R); i += 256) tab[i] = bias_value(rel, R, h, i - kBiasPad);
}

// The block's unit and head (see placed()); a unit past the last one has no work.
__device__ __forceinline__ void place(int chunk, int heads, int& unit, int& head) {
  const int b = blockIdx.x;
  if (chunk) {
    const int i = b >> 3, x = b & 7;
    head = x & (heads - 1);
    unit = (i / chunk * (8 / heads) + x / heads) * chunk + i % chunk;
  } else {
    head = b % heads;
    unit = b / heads;
  }
}

// The unit's group, and its number within it.
template <bool KEYS>
__device__ __forceinline__ TrainGroup group_of(const TrainArgs& a, int unit, int lane, int& local) {
  const uint32_t* const order = KEYS ? a.k_order : a.q_order;
  if (order) {
    const uint32_t x = order[unit];
    local = x >> 16;
    return a.groups[x & 0xffff];
  }
  const TrainGroup g = a.groups[find_group<KEYS>(a.groups, a.n_groups, unit, lane)];
  local = unit - (KEYS ? g.unit_k : g.unit_q);
  return g;
}

// Lets a kernel use more than 64 KB of LDS a block: remembers the most that it
// was allowed on each device, and never lowers it.
struct LdsAllowed {
  std::mutex mu;
  size_t bytes[64] = {};
};
inline hipError_t allow_lds(const void* kernel, size_t bytes, LdsAllowed& so_far) {
  if (bytes <= 65536) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(so_far.mu);
  if (so_far.bytes[dev] >= bytes) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == hipSuccess) so_far.bytes[dev] = bytes;
  return e;
}

#endif  // __HIPCC__

}  // namespace tx
