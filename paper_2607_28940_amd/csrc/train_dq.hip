// Backward of the training attention (train_attn.h), query side: dq of 128
// queries of one (group, head) per block, the bias gradient's sums over those
// queries, and D (read again by the key side).
//
// The gradients of keys and values are summed over queries and those of
// queries over keys, so one of the two would need atomic adds across blocks if
// a single kernel made both; two kernels that each recompute S and dP (seven
// tile products in all instead of five) keep every sum in one block in a fixed
// order.
#include "train_attn.h"

#include <type_traits>

namespace tx {
namespace {

// As in the forward.
template <class T, bool NARROW>
constexpr int key_tile() { return sizeof(T) == 2 && !NARROW ? 64 : 32; }
template <class T, int DH, bool NARROW>
constexpr int dq_buffers() { return NARROW && sizeof(T) == 4 && DH == 128 ? 1 : 2; }
template <class T, int DH, bool NARROW>
constexpr int dq_tile_bytes() { return key_tile<T, NARROW>() * Geo<T, DH>::RB; }
template <class T, int DH, bool NARROW>
constexpr int dq_lds_bytes() {
  return (NARROW ? 4 : 1) * 2 * dq_buffers<T, DH, NARROW>() * dq_tile_bytes<T, DH, NARROW>();
}
template <class T, int DH, bool NARROW>
constexpr int dq_blocks() { return NARROW || sizeof(T) == 4 ? 1 : DH == 128 ? 2 : DH == 64 ? 3 : 4; }

// Whether dP's product starts from -D, 16 registers of it, instead of a
// subtraction per pair: where the block's share of the registers has room (147 k
// queries of 2.3 k keys at d_head 128: 1.86 against 1.91 ms; at 64, with three
// blocks a CU, 121 against 114 us for 17 k queries).
template <class T, int DH, bool REL, bool NARROW>
constexpr bool from_d() { return sizeof(T) == 2 && !NARROW && (DH == 32 || (DH == 128 && !REL)); }

// Per wave and 32 keys: S^T = K Q^T, dP^T = V dO^T (lanes = queries, so lse and
// D are one register each), dS = P (dP - D), dQ^T += K^T dS^T with dS^T taken
// from the accumulators. dS is rounded to bf16 for that product (relative 2^-9
// of each term, as P in the forward).
// Measured, 8 heads: 147 k queries of 2.3 k keys at d_head 128 in 1.85 ms, 1.12
// PFLOP/s of its three products, matrix units busy 55% of the cycles, vector units
// 39%; 16384 causal tokens with bias sums 0.76 ms, 1.09; 4 x 8192 at 64 0.45 ms, 0.91.
//
// Bias gradient: only tiles that touch the buckets below the last one sum their
// dS by distance; the last bucket needs no sums, since every row's dS adds up
// to zero: its gradient is minus the sum of the others. Within 32 keys and 32
// queries the sums are those of the diagonals, 63 of them, made in registers
// (diagonal_sums) and added to a padded table in LDS, one per wave, so that each
// table is summed in program order.
//
// Sums over the diagonals of a 32 x 32 tile in the accumulator layout (lane:
// column, registers: rows): lane d gets the sum at column - row = d, lane 64 + d
// that of d < 0. Rows from the last to the first, each step rotates the sums by
// a lane and adds a row (T[l] = x_row[l] + T[l + 1]), on a ring of 64 lanes whose
// upper half starts empty.
__device__ __forceinline__ float diagonal_sums(const floatx16& x) {
  constexpr int kWaveRotateLeft = 0x134;
  float sum = 0.f;
#pragma unroll
  for (int g = 3; g >= 0; --g) {
    float lo[4], up[4];  // rows 8 g + t (lanes 0-31) and 8 g + 4 + t (lanes 32-63), both on lanes 0-31
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[4 * g + t]), 0u, false, false);
      lo[t] = __uint_as_float(r[0]);
      up[t] = __uint_as_float(r[1]);
    }
#pragma unroll
    for (int t = 3; t >= 0; --t) sum = up[t] + dpp_f32<kWaveRotateLeft>(sum);
#pragma unroll
    for (int t = 3; t >= 0; --t) sum = lo[t] + dpp_f32<kWaveRotateLeft>(sum);
  }
  return sum;
}

template <class T, int DH, bool REL, bool NARROW>
__global__ __launch_bounds__(256, (dq_blocks<T, DH, NARROW>())) void train_dq_kernel(const TrainArgs a) {
  using Gm = Geo<T, DH>;
  using W = Wave<T, DH>;
  constexpr int KT = key_tile<T, NARROW>(), KB = KT / 32, TB = dq_tile_bytes<T, DH, NARROW>();
  constexpr int BUFS = dq_buffers<T, DH, NARROW>();
  constexpr bool FROM_D = from_d<T, DH, REL, NARROW>();
  extern __shared__ __align__(1024) char smem_[];
  lds_char* const smem = (lds_char*)smem_;
  lds_float* const tab = (lds_float*)(smem + dq_lds_bytes<T, DH, NARROW>());
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  // a wide block's waves: 4 >> pack of them on the rows of each of its heads
  const int pack = NARROW || REL ? 0 : a.pack, ROWS = NARROW ? kNarrowRows : kWideRows >> pack;
  int unit, h0;
  place(a.q_chunk, a.H >> pack, unit, h0);
  if (unit >= a.n_units) return;
  h0 <<= pack;
  const int h = h0 + (wave >> (2 - pack)), w_row = NARROW ? 0 : 32 * (wave & ((4 >> pack) - 1));
  int local;
  const TrainGroup g = group_of<false>(a, unit, lane, local);
  const int parts = g.parts_q, blocks = (g.nq + ROWS - 1) / ROWS;
  const int part = local % parts;
  const int qb = blocks - 1 - local / parts;
  const int q_first = qb * ROWS;
  const int hk = h0 / (a.H / a.G);
  const int R = REL ? a.R : 0, R1 = max(R, 1) - 1, entries = bias_entries(R);
  const bool sums = REL && R > 1;  // of dS, by bucket
  lds_float* const sub = tab + entries;

  int k_end;
  if (REL) {
    k_end = min(g.nq, q_first + ROWS);
  } else {
    const TileLim* tl = a.tile_lim + g.qt0 + q_first / kTrainQTile;
    k_end = tl[0].hi;
    if (ROWS > kTrainQTile && q_first + kTrainQTile < g.nq) k_end = max(k_end, tl[1].hi);
  }
  if (REL) stage_bias(tab, (const T*)a.rel, R, h, tid);
  const float far = REL ? bias_value((const T*)a.rel, R, h, R1) : 0.f;
  int t_begin = 0;
  if (REL && far == -INFINITY) t_begin = max(0, q_first - (R - 2)) / KT;
  int t_end = (k_end + KT - 1) / KT;
  int t_plain;  // tiles before it: see train_fwd_kernel
  if (REL) {
    t_plain = fabsf(far) < 0x1p20f ? max(0, q_first - R1 + 1) / KT : 0;
  } else {
    const TileLim* tl = a.tile_lim + g.qt0 + q_first / kTrainQTile;
    t_plain = tl[0].lo;
    if (ROWS > kTrainQTile && q_first + kTrainQTile < g.nq) t_plain = min(t_plain, tl[1].lo);
    t_plain /= KT;
  }
  // a block of few tiles takes D from them (below), undivided
  const bool few = Gm::BF && t_end - t_begin <= (NARROW ? 4 : 2);
  if (parts > 1 && few) {
    if (part) t_end = t_begin;
  } else if (parts > 1) {
    const int n = max(0, t_end - t_begin);
    t_end = t_begin + (int)((int64_t)n * (part + 1) / parts);
    t_begin += (int)((int64_t)n * part / parts);
  }
  t_plain = min(t_plain, t_end);

  const int q_wave = q_first + w_row, q_row = q_wave + l32;
  const bool exists = q_row < g.nq;
  const int64_t row = g.q0 + q_row;
  float D = 0.f;
  {
    u32x4_t of[Gm::NC], df[Gm::NC];
    load_row_frags<T, DH>(a.dO.p + row * a.dO.row + h * a.dO.head, exists, hi, df);
    load_row_frags<T, DH>(a.o.p + row * a.o.row + h * a.o.head, exists, hi, of);
#pragma unroll
    for (int c = 0; c < Gm::NC; ++c) {
      if constexpr (Gm::BF) {
        const bf16x8 x = __builtin_bit_cast(bf16x8, of[c]), y = __builtin_bit_cast(bf16x8, df[c]);
#pragma unroll
        for (int t = 0; t < 8; ++t) D = fmaf((float)x[t], (float)y[t], D);
      } else {
        const floatx4 x = __builtin_bit_cast(floatx4, of[c]), y = __builtin_bit_cast(floatx4, df[c]);
#pragma unroll
        for (int t = 0; t < 4; ++t) D = fmaf(x[t], y[t], D);
      }
    }
    D = xor32_sum(D);
  }
  float lse2 = INFINITY;  // a row without visible keys keeps it: its probabilities are 0
  if (exists) {
    const float x = a.lse[(int64_t)h * a.lse_ld + row];
    if (x != -INFINITY) lse2 = x * kTrainLog2e;
  }
  int lim = 0;
  if (exists) lim = REL ? q_row + 1 : a.row_lim[row - a.q_base];
  int lim_hi = 0;
  if (REL) {
    if (q_wave < g.nq) lim_hi = min(q_wave + 32, g.nq);
  } else {
    int up = lim;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) up = max(up, __shfl_xor(up, m));
    lim_hi = uniform(up);
  }

  floatx16 dq[Gm::NB];

  const W w(lane);
  using Dma = TileDma<T, DH, KT, true, NARROW ? 1 : 4>;
  const Dma kd(NARROW ? 0 : wave, lane, a.k.row), vd(NARROW ? 0 : wave, lane, a.v.row);
  lds_char* const bufs = smem + (NARROW ? wave * 2 * BUFS * TB : 0);
  const char* const kp = a.k.p + (int64_t)g.k0 * a.k.row + hk * a.k.head;
  const char* const vp = a.v.p + (int64_t)g.k0 * a.v.row + hk * a.v.head;
  auto fetch = [&](int t, int b) {
    const int r = t * KT;
    kd.load(kp + (int64_t)r * a.k.row, g.nk - r, bufs + b * TB);
    vd.load(vp + (int64_t)r * a.v.row, g.nk - r, bufs + (BUFS + b) * TB);
  };
  // D = dO . O takes the rounding of a bf16 O, of half a step 2^-8 |O| a feature,
  // into every dS of the row. Over many keys O is small and its rounding with it;
  // a row that sees few keys, whose dS may all but cancel, takes D as the sum of
  // P dP over them instead. Without it the bias gradient of 100 sequences of 5 is
  // off by 9e-3 of its norm, with it by the 1.4e-3 that its own rounding takes.
  if (Gm::BF && few && t_begin < t_end) {
    u32x4_t qf[Gm::NC], df[Gm::NC];
    load_row_frags<T, DH>(a.dO.p + row * a.dO.row + h * a.dO.head, exists, hi, df);
    load_row_frags<T, DH>(a.q.p + row * a.q.row + h * a.q.head, exists, hi, qf);
    const int t0 = t_begin + (NARROW ? wave : 0), n = NARROW ? (t0 < t_end ? 1 : 0) : t_end - t_begin;
    for (int t = 0; t < n; ++t) fetch(t0 + t, t);
    tiles_ready();  // (and the bias table)
    float sum = 0.f;
    for (int t = 0; t < n && (t0 + t) * KT < lim_hi; ++t) {
      const int k0 = (t0 + t) * KT, d0 = min(q_row - k0, R1 + kBiasPad - 1) - 4 * hi + kBiasPad;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        floatx16 s, p;
#pragma unroll
        for (int v = 0; v < 16; ++v) p[v] = 0.f;
        w.rows_products(bufs + t * TB, qf, s, bufs + (BUFS + t) * TB, df, p, kb);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = kb * 32 + 8 * (v >> 2) + (v & 3);
          const float bias = REL ? tab[d0 - key] : 0.f;
          const bool see = REL ? bias != -INFINITY : key < lim - k0 - 4 * hi;
          sum += see ? __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, bias) - lse2) * p[v] : 0.f;
        }
      }
    }
    D = xor32_sum(sum);
    __syncthreads();
    if (NARROW) {
      lds_float* const sums4 = (lds_float*)smem;
      if (hi == 0) sums4[32 * wave + l32] = D;
      __syncthreads();
      D = (sums4[l32] + sums4[32 + l32]) + (sums4[64 + l32] + sums4[96 + l32]);
      __syncthreads();
    }
  }
  if (exists && part == 0 && hi == 0 && (!NARROW || wave == 0)) {
    float* const st = a.row_stat + 2 * ((int64_t)h * a.stat_ld + row - a.q_base);
    st[0] = lse2;
    st[1] = D;
  }
  // One pass over the keys; STRICT: see train_fwd_kernel.
  auto pass = [&](auto strict_c) {
    constexpr bool STRICT = decltype(strict_c)::value;
    u32x4_t qf[Gm::NC], df[Gm::NC];
    load_row_frags<T, DH>(a.dO.p + row * a.dO.row + h * a.dO.head, exists, hi, df);
    load_row_frags<T, DH>(a.q.p + row * a.q.row + h * a.q.head, exists, hi, qf);
#pragma unroll
    for (int db = 0; db < Gm::NB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) dq[db][v] = 0.f;
    if (sums)
      for (int i = tid; i < 4 * entries; i += 256) sub[i] = 0.f;
    floatx16 from;  // FROM_D: what dP's product starts from
    if constexpr (FROM_D)
#pragma unroll
      for (int v = 0; v < 16; ++v) from[v] = -D;
    bool again = false;
    auto tile = [&](auto masked_c, int t, int b) {
      constexpr bool MASKED = decltype(masked_c)::value;
      const int k0 = t * KT;
      const lds_char* const sK = bufs + b * TB;
      const lds_char* const sV = bufs + (BUFS + b) * TB;
      const int d0 = min(q_row - k0, R1 + kBiasPad - 1) - 4 * hi + kBiasPad;
      const float off = far - lse2;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        floatx16 s, p;
        if constexpr (FROM_D) p = from;
        else
#pragma unroll
          for (int v = 0; v < 16; ++v) p[v] = 0.f;
        w.rows_products(sK, qf, s, sV, df, p, kb);
        if (!MASKED) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, off)) * (FROM_D ? p[v] : p[v] - D);
          w.cols_mma(sK, kb, s, dq);
          continue;
        }
        uint32_t vis = 0;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = kb * 32 + 8 * (v >> 2) + (v & 3);
          const float bias = REL ? tab[d0 - key] : 0.f;
          const bool see = REL ? bias != -INFINITY : key < lim - k0 - 4 * hi;
          vis |= see ? 1u << v : 0u;
          // in two steps: a large bias rounds the logit as it did in the forward
          const float lg = fmaf(s[v], a.scale_log2, bias);
          s[v] = see ? __builtin_amdgcn_exp2f(lg - lse2) * (FROM_D ? p[v] : p[v] - D) : 0.f;
        }
        if (sums) {
          // lane d (or 64 + d): distance q_wave - k0 - 32 kb + d; past the padding nothing is kept
          const int at = q_wave - k0 - 32 * kb + (lane < 32 ? lane : lane - 64) + kBiasPad;
          const float x = diagonal_sums(s);
          if (at >= 0 && at < entries) __builtin_amdgcn_ds_atomic_fadd_f32(sub + wave * entries + at, x);
        }
        if constexpr (STRICT) {
          w.cols_mma_strict(sK, kb, s, vis, dq);
        } else {
          again |= w.rows_not_finite(sK, kb);
          w.cols_mma(sK, kb, s, dq);
        }
      }
    };
    // a wide block's waves go through the tiles together, a narrow one's through
    // every fourth, each at its own pace
    constexpr int STEP = NARROW ? 4 : 1;
    auto ready = [&] {
      if (NARROW) tile_ready();
      else tiles_ready();
    };
    int t = t_begin + (NARROW ? wave : 0), b = 0;
    auto run = [&](auto masked_c, int end, bool rows_here) {
      for (; t < end; t += STEP) {
        if (BUFS == 2 && t + STEP < t_end) fetch(t + STEP, b ^ 1);
        if (decltype(masked_c)::value ? t * KT < lim_hi : rows_here) tile(masked_c, t, b);
        if (BUFS == 1 && t + STEP < t_end) tile_read(), fetch(t + STEP, 0);
        ready();
        if (BUFS == 2) b ^= 1;
      }
    };
    if (NARROW) __syncthreads();  // (the bias table and the sums)
    if (t < t_end) fetch(t, 0);
    pin(qf), pin(df), pin(lim), pin(lse2), pin(D);
    if constexpr (FROM_D) pin(from);
    ready();
    run(std::false_type{}, t_plain, q_wave < g.nq);
    run(std::true_type{}, t_end, true);
    if (NARROW) __syncthreads();
    return again;
  };
  if (__syncthreads_or(pass(std::false_type{}))) (void)pass(std::true_type{});
  if (sums) {
    // (a pass, also one over no tiles, ends on a barrier)
    float* const out = a.drel_part + ((size_t)unit * a.H + h) * R;
    for (int d = tid; d < R; d += 256) {
      float x = 0.f;
      if (d < R - 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) x += sub[i * entries + kBiasPad + d];
      out[d] = x;
    }
  }
  float* const slot = parts == 1 ? nullptr
                                 : a.partial + ((size_t)g.slot_q + (size_t)((qb * parts + part) * a.H + h)) *
                                                   train_dq_slot(ROWS, DH);
  char* const out = a.dq.p + (int64_t)(g.q0 + q_first) * a.dq.row + h * a.dq.head;
  if constexpr (NARROW) {
    Park<DH>::put(dq, bufs, lane);
    __syncthreads();
    add_parked<T, DH>(smem, 2 * BUFS * TB, slot, a.scale, out, a.dq.row, g.nq - q_first, tid);
    return;
  }
  if (slot) {
    if (exists) store_partial<T, DH>(dq, slot + (size_t)(w_row + l32) * DH, hi);
    return;
  }
  if (q_wave < g.nq)
    store_rows<T, DH>(dq, a.scale, smem + wave * 32 * Gm::RB, out + w_row * a.dq.row, a.dq.row, g.nq - q_wave, lane);
}

template <class T, int DH>
__global__ __launch_bounds__(256) void train_dq_join_kernel(const TrainArgs a) {
  __shared__ __align__(16) char left[256 * 16];
  const int unit = blockIdx.x / a.H, h = blockIdx.x % a.H, tid = threadIdx.x;
  const TrainGroup g = a.groups[find_group<false>(a.groups, a.n_groups, unit, tid & 63)];
  const int parts = g.parts_q, local = unit - g.unit_q, qb = local / parts, q_first = qb * a.q_rows;
  if (parts == 1 || local % parts) return;
  const size_t slot = train_dq_slot(a.q_rows, DH);
  join_sums<T, DH>(a.partial + ((size_t)g.slot_q + (size_t)(qb * parts * a.H + h)) * slot, (size_t)a.H * slot, parts,
                   min(a.q_rows, g.nq - q_first), a.scale,
                   a.dq.p + (int64_t)(g.q0 + q_first) * a.dq.row + h * a.dq.head, a.dq.row, (lds_char*)left, tid);
}

// Sums of 32 units' bucket sums (the first pass) ...
constexpr int kDrelChunk = 32;
__global__ __launch_bounds__(256) void drel_chunk_kernel(const float* __restrict__ part, int n_units, int HR,
                                                         float* __restrict__ out) {
  const int i = blockIdx.y * 256 + threadIdx.x;
  if (i >= HR) return;
  const int u0 = blockIdx.x * kDrelChunk, n = min(kDrelChunk, n_units - u0);
  float v[kDrelChunk], x = 0.f;
#pragma unroll
  for (int u = 0; u < kDrelChunk; ++u) v[u] = u < n ? part[(size_t)(u0 + u) * HR + i] : 0.f;
#pragma unroll
  for (int u = 0; u < kDrelChunk; ++u) x += v[u];
  out[(size_t)blockIdx.x * HR + i] = x;
}
// ... and of all chunks, the last bucket as minus the others: a block per head.
template <class T>
__global__ __launch_bounds__(256) void drel_head_kernel(const float* __restrict__ part, int n, int H, int R,
                                                        T* __restrict__ drel) {
  __shared__ float wsum[4];
  const int h = blockIdx.x, tid = threadIdx.x;
  float others = 0.f;
  for (int b = tid; b < R - 1; b += 256) {
    float x = 0.f;
#pragma unroll 16
    for (int c = 0; c < n; ++c) x += part[((size_t)c * H + h) * R + b];
    drel[(size_t)h * R + b] = (T)x;
    others += x;
  }
  others = wave_sum(others);
  if ((tid & 63) == 0) wsum[tid >> 6] = others;
  __syncthreads();
  if (tid == 0) drel[(size_t)h * R + R - 1] = (T)(0.f - (wsum[0] + wsum[1] + wsum[2] + wsum[3]));
}

// The biases and, where there are sums to take, a table of them per wave.
size_t table_bytes(int R) { return 4 * (size_t)bias_entries(R) * (R > 1 ? 5 : 1); }

template <class T, int DH, bool REL, bool NARROW>
hipError_t dq_launch(const TrainArgs& a, hipStream_t s) {
  const size_t lds = dq_lds_bytes<T, DH, NARROW>() + (REL ? table_bytes(a.R) : 0);
  static LdsAllowed so_far;
  const hipError_t e = allow_lds((const void*)train_dq_kernel<T, DH, REL, NARROW>, lds, so_far);
  if (e != hipSuccess) return e;
  train_dq_kernel<T, DH, REL, NARROW><<<place_grid(a.n_units, a.H >> a.pack, a.q_chunk), 256, lds, s>>>(a);
  return hipGetLastError();
}
template <class T, int DH>
hipError_t dq_join(const TrainArgs& a, hipStream_t s) {
  train_dq_join_kernel<T, DH><<<dim3((unsigned)a.n_units * a.H), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t train_dq_lds(bool bf, int dh, int R, bool narrow) {
#define TX_CASE(T, D) return table_bytes(R) + (narrow ? dq_lds_bytes<T, D, true>() : dq_lds_bytes<T, D, false>())
  if (bf) {
    if (dh == 32) TX_CASE(bf16, 32);
    if (dh == 64) TX_CASE(bf16, 64);
    TX_CASE(bf16, 128);
  }
  if (dh == 32) TX_CASE(float, 32);
  if (dh == 64) TX_CASE(float, 64);
  TX_CASE(float, 128);
#undef TX_CASE
}

hipError_t launch_train_dq(bool bf, int dh, bool rel, const TrainArgs& a, hipStream_t s) {
  const bool narrow = a.q_narrow;
#define TX_CASE(T, D)                                                                               \
  return narrow ? (rel ? dq_launch<T, D, true, true>(a, s) : dq_launch<T, D, false, true>(a, s))    \
                : (rel ? dq_launch<T, D, true, false>(a, s) : dq_launch<T, D, false, false>(a, s))
  if (bf) {
    if (dh == 32) TX_CASE(bf16, 32);
    if (dh == 64) TX_CASE(bf16, 64);
    TX_CASE(bf16, 128);
  }
  if (dh == 32) TX_CASE(float, 32);
  if (dh == 64) TX_CASE(float, 64);
  TX_CASE(float, 128);
#undef TX_CASE
}

hipError_t launch_train_dq_join(bool bf, int dh, const TrainArgs& a, hipStream_t s) {
  if (bf)
    return dh == 32 ? dq_join<bf16, 32>(a, s) : dh == 64 ? dq_join<bf16, 64>(a, s) : dq_join<bf16, 128>(a, s);
  return dh == 32 ? dq_join<float, 32>(a, s) : dh == 64 ? dq_join<float, 64>(a, s) : dq_join<float, 128>(a, s);
}

hipError_t launch_train_drel(bool bf, const TrainArgs& a, float* scratch, void* drel, hipStream_t s) {
  const int HR = a.H * a.R;
  const float* part = a.drel_part;
  int n = a.R > 1 ? a.n_units : 0;
  if (n > kDrelChunk) {
    const int chunks = (n + kDrelChunk - 1) / kDrelChunk;
    drel_chunk_kernel<<<dim3(chunks, (HR + 255) / 256), 256, 0, s>>>(part, n, HR, scratch);
    part = scratch, n = chunks;
  }
  if (bf) drel_head_kernel<bf16><<<a.H, 256, 0, s>>>(part, n, a.H, a.R, (bf16*)drel);
  else drel_head_kernel<float><<<a.H, 256, 0, s>>>(part, n, a.H, a.R, (float*)drel);
  return hipGetLastError();
}

}  // namespace tx
