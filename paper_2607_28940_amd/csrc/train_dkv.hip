// Backward of the training attention (train_attn.h), key side: dk and dv of 128
// keys of one (group, key head) per block, summed over the queries of every
// query head that reads the key head. Keys that no query sees get zeros.
#include "train_attn.h"

#include <type_traits>

namespace tx {
namespace {

// Whether the block's V rows stay in LDS instead of registers: at d_head 128 the
// accumulators of dk and dv (128 registers), the K and V fragments (64) and a
// tile's S and dP do not fit 256 registers, and every spill waits for the tiles
// in flight. In bf16, V in LDS with 32-row tiles keeps two blocks on a CU (66 KB
// each): 17.8 -> 4.1 ms for 147 k queries of 2.3 k keys on average. At d_head 64
// V in LDS lets three blocks of 168 registers share a CU (1.16 against 1.24 ms
// for 111 k queries of 2.3 k keys with two), at 32 it fits registers four times
// over. A narrow block has its CU to itself.
template <class T, int DH, bool NARROW>
constexpr bool v_in_lds() { return sizeof(T) == 2 && DH >= 64 && !NARROW; }
// Rows of a query tile, tile buffers (Q and dO each) of a block or of a narrow
// block's wave, bytes of a tile, and bytes of all tiles and V.
template <class T, int DH, bool NARROW>
constexpr int query_tile() { return sizeof(T) == 2 && DH < 128 && !NARROW ? 64 : 32; }
template <class T, int DH, bool NARROW>
constexpr int dkv_buffers() { return NARROW && sizeof(T) == 4 && DH == 128 ? 1 : 2; }
template <class T, int DH, bool NARROW>
constexpr int dkv_tile_bytes() { return query_tile<T, DH, NARROW>() * Geo<T, DH>::RB; }
template <class T, int DH, bool NARROW>
constexpr int dkv_lds_bytes() {
  return (NARROW ? 4 : 1) * 2 * dkv_buffers<T, DH, NARROW>() * dkv_tile_bytes<T, DH, NARROW>() +
         (v_in_lds<T, DH, NARROW>() ? kWideRows * Geo<T, DH>::RB : 0);
}
// Row statistics: [2 buffers][lse, D, limits][rows of a tile] of a block or of
// each wave.
template <class T, int DH, bool NARROW>
constexpr int stat_floats() { return (NARROW ? 4 : 1) * 6 * query_tile<T, DH, NARROW>(); }
template <class T, int DH, bool NARROW>
constexpr int dkv_blocks() { return NARROW || sizeof(T) == 4 ? 1 : DH == 128 ? 2 : DH == 64 ? 3 : 4; }

// A wave owns 32 keys, whose K (and V) fragments stay in registers. Per 32
// queries: S = Q K^T and dP = dO V^T (lanes = keys), P and dS = P (dP - D),
// then dV^T += dO^T P and dK^T += Q^T dS with P and dS taken from the
// accumulators and the columns of the dO and Q tiles read from LDS (bf16:
// transposing reads). P and dS are rounded to bf16 for those products. Q, dO
// and the rows' lse, D and key limits are double-buffered, one barrier a tile.
// Measured, 8 heads: 147 k queries of 2.3 k keys at d_head 128 in 3.0 ms, 0.93
// PFLOP/s of its four products, matrix units busy 46% of the cycles, the LDS a
// third, barriers and LDS latency most of the rest (256 registers, two waves a
// SIMD); 16384 causal tokens 1.14 ms, 0.97; 4 x 8192 at 64 0.63 ms, 0.88.
template <class T, int DH, bool REL, bool NARROW>
__global__ __launch_bounds__(256, (dkv_blocks<T, DH, NARROW>())) void train_dkv_kernel(const TrainArgs a) {
  using Gm = Geo<T, DH>;
  using W = Wave<T, DH>;
  constexpr int QT = query_tile<T, DH, NARROW>(), QB = QT / 32, TB = dkv_tile_bytes<T, DH, NARROW>();
  constexpr int BUFS = dkv_buffers<T, DH, NARROW>(), ROWS = NARROW ? kNarrowRows : kWideRows, STEP = NARROW ? 4 : 1;
  constexpr bool V_LDS = v_in_lds<T, DH, NARROW>();
  extern __shared__ __align__(1024) char smem_[];
  lds_char* const smem = (lds_char*)smem_;
  lds_char* const sVb = smem + 2 * BUFS * TB;  // V_LDS: the block's V rows
  lds_float* const stats = (lds_float*)(smem + dkv_lds_bytes<T, DH, NARROW>());
  lds_float* const tab = stats + stat_floats<T, DH, NARROW>();
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  int unit, hk;
  place(a.k_chunk, a.G, unit, hk);
  if (unit >= a.k_units) return;
  const int per = a.H / a.G;
  int local;
  const TrainGroup g = group_of<true>(a, unit, lane, local);
  const int parts = g.parts_k, part = local % parts, kblk = local / parts;
  const int k_first = kblk * ROWS, k_wave = k_first + (NARROW ? 0 : wave * 32), key = k_wave + l32;
  lds_char* const bufs = smem + (NARROW ? wave * 2 * BUFS * TB : 0);
  lds_float* const stat = stats + (NARROW ? wave * 6 * QT : 0);
  const bool exists = key < g.nk;
  const int R = REL ? a.R : 0;

  floatx16 dk[Gm::NB], dv[Gm::NB];

  // Work list of the block: (query head, query tile), heads outermost. Causal
  // rows before the block's first key do not see it.
  const int nqt = (g.nq + QT - 1) / QT, t0 = REL ? min(nqt, k_first / QT) : 0, per_head = nqt - t0;
  int i0 = 0, i1 = per * per_head;
  if (parts > 1) {
    const int n = i1;
    i1 = (int)((int64_t)n * (part + 1) / parts);
    i0 = (int)((int64_t)n * part / parts);
  }
  const int R1 = max(R, 1) - 1, k_last = min(g.nk, k_first + ROWS) - 1;
  // causal tiles from t_far on have one bias, the last bucket's
  const int t_far = REL ? (k_last + R1 + QT - 1) / QT : 0;
  float far = 0.f;  // the head's last bucket
  // Classes of query tiles: 2 plain (every row sees every key of the block, one
  // bias), 1 masked or with biases of its own, 0 sees nothing.
  auto tile_class = [&](int t) { return t < t_far ? 1 : far == -INFINITY ? 0 : fabsf(far) < 0x1p20f ? 2 : 1; };
  auto limit_class = [&](int t) {
    const TileLim x = a.tile_lim[g.qt0 + t];
    return x.hi <= k_first ? 0 : x.lo > k_last ? 2 : 1;
  };
  using Dma = TileDma<T, DH, QT, !V_LDS, NARROW ? 1 : 4>;
  const Dma qd(NARROW ? 0 : wave, lane, a.q.row), dd(NARROW ? 0 : wave, lane, a.dO.row);
  // The rows' statistics: threads (a narrow block's lanes) 0 .. QT - 1 fetch lse and D, the next QT the
  // limits, with the tile (rows past the last one read the last); they are parked
  // in LDS once the tile before has been computed, and nothing touches them till
  // then, as that would wait for the tile too.
  typedef float float2_t __attribute__((ext_vector_type(2)));
  auto fetch_stat = [&](int h, int t) {
    int id = NARROW ? lane : tid;
    asm volatile("" : "+v"(id));  // not hoisted
    const int64_t r = g.q0 + min(t * QT + id % QT, g.nq - 1) - a.q_base;
    const float2_t* p = (const float2_t*)a.row_stat + (h * a.stat_ld + r);
    if (!REL && id >= QT) p = (const float2_t*)(a.row_lim + (r & ~1));
    return *p;
  };
  // in the form that the tiles of the class take: plain ones the negative lse and
  // their bias together, both minus D, which dP's product starts from
  auto park_stat = [&](auto masked_c, float2_t x, int t, int b) {
    int id = NARROW ? lane : tid;
    asm volatile("" : "+v"(id));
    const int r = t * QT + id % QT;
    const bool ok = r < g.nq;
    lds_float* const to = stat + b * 3 * QT + id;
    if (id < QT) {
      const float ls = ok ? x[0] : INFINITY;  // (probabilities 0)
      to[0] = decltype(masked_c)::value ? ls : far - ls;
      to[QT] = ok ? -x[1] : 0.f;
    } else if (!REL && id < 2 * QT) {
      to[QT] = ok ? ((g.q0 + r - a.q_base) & 1 ? x[1] : x[0]) : 0.f;
    }
  };
  auto fetch = [&](int h, int t, int b) {
    const int r = t * QT;
    qd.load(a.q.p + (int64_t)(g.q0 + r) * a.q.row + h * a.q.head, g.nq - r, bufs + b * TB);
    dd.load(a.dO.p + (int64_t)(g.q0 + r) * a.dO.row + h * a.dO.head, g.nq - r, bufs + (BUFS + b) * TB);
  };
  // One pass over the work list; STRICT: see train_fwd_kernel.
  auto pass = [&](auto strict_c) {
    constexpr bool STRICT = decltype(strict_c)::value;
    u32x4_t kf[Gm::NC], vf[V_LDS ? 1 : Gm::NC];
    load_row_frags<T, DH>(a.k.p + (int64_t)(g.k0 + key) * a.k.row + hk * a.k.head, exists, hi, kf);
    if constexpr (V_LDS) {
      const TileDma<T, DH, kWideRows, false> vd(wave, lane, a.v.row);
      vd.load(a.v.p + (int64_t)(g.k0 + k_first) * a.v.row + hk * a.v.head, g.nk - k_first, sVb);
    } else {
      load_row_frags<T, DH>(a.v.p + (int64_t)(g.k0 + key) * a.v.row + hk * a.v.head, exists, hi, vf);
    }
#pragma unroll
    for (int db = 0; db < Gm::NB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) dk[db][v] = 0.f, dv[db][v] = 0.f;
    pin(kf);
    if (!V_LDS) pin(vf);
    bool again = false;
    auto tile = [&](auto masked_c, int t, int b) {
      constexpr bool MASKED = decltype(masked_c)::value;
      const lds_char* const sQ = bufs + b * TB;
      const lds_char* const sO = bufs + (BUFS + b) * TB;
      const lds_float* const ss = stat + b * 3 * QT;
      // at d_head 128 the fragments' addresses are cheaper made anew than held
      int id = NARROW ? lane : tid;
      if (V_LDS) asm volatile("" : "+v"(id));  // not hoisted
      const W w(id & 63);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int qr = t * QT + 32 * qb;  // first query of the 32
        if (MASKED && (qr >= g.nq || (REL && qr + 31 < k_wave))) continue;
        floatx16 s, p;
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
          const floatx4 nD = *reinterpret_cast<const lds_floatx4*>(ss + QT + 32 * qb + 8 * gq + 4 * hi);
#pragma unroll
          for (int t = 0; t < 4; ++t) p[4 * gq + t] = nD[t];
        }
        if constexpr (V_LDS) w.rows_products_lds(sQ, kf, s, sO, sVb + wave * 32 * Gm::RB, p, qb);
        else w.template rows_products<4>(sQ, kf, s, sO, vf, p, qb);
        if (!MASKED) {
#pragma unroll
          for (int gq = 0; gq < 4; ++gq) {
            const floatx4 ls = *reinterpret_cast<const lds_floatx4*>(ss + 32 * qb + 8 * gq + 4 * hi);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const int v = 4 * gq + t;
              s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, ls[t]));
              p[v] *= s[v];
            }
          }
          w.cols_mma2(sO, s, dv, sQ, p, dk, qb);
          continue;
        }
        const int d0 = min(qr - key, R1 + kBiasPad - 32) + 4 * hi + kBiasPad;
        uint32_t vis = 0;
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
          const floatx4 ls = *reinterpret_cast<const lds_floatx4*>(ss + 32 * qb + 8 * gq + 4 * hi);
          floatx4 lm = {0.f, 0.f, 0.f, 0.f};
          if (!REL) lm = *reinterpret_cast<const lds_floatx4*>(ss + 2 * QT + 32 * qb + 8 * gq + 4 * hi);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int v = 4 * gq + t;
            const float bias = REL ? tab[d0 + 8 * gq + t] : 0.f;
            const bool see = REL ? bias != -INFINITY : key < __float_as_int(lm[t]);
            vis |= see ? 1u << v : 0u;
            const float lg = fmaf(s[v], a.scale_log2, bias);
            s[v] = see ? __builtin_amdgcn_exp2f(lg - ls[t]) : 0.f;
            p[v] = see ? s[v] * p[v] : 0.f;
          }
        }
        if constexpr (STRICT) {
          w.cols_mma_strict(sO, qb, s, vis, dv);
          w.cols_mma_strict(sQ, qb, p, vis, dk);
        } else {
          again |= w.rows_not_finite(sO, qb) | w.rows_not_finite(sQ, qb);
          w.cols_mma2(sO, s, dv, sQ, p, dk, qb);
        }
      }
    };
    // The tiles of one class of the heads hh .. h1 - 1, the next one on its way
    // while one is computed; a narrow block's wave takes every fourth of them, by
    // itself. MANY: more heads than one may follow each other.
    auto run = [&](auto masked_c, auto many_c, int hh, int h1) {
      constexpr int CLASS = decltype(masked_c)::value ? 1 : 2;
      constexpr bool MANY = decltype(many_c)::value;
      int t, t1;
      // causal classes go by the tile's index, event ones by a mask over 64 limit
      // tiles that the wave looks at together
      int m0 = -64;
      uint64_t mask = 0;
      auto head = [&] {  // the head's share of the work list
        t = t0 + max(0, i0 - hh * per_head);
        t1 = t0 + min(per_head, i1 - hh * per_head);
        if (REL && CLASS == 2) t = max(t, t_far);
        if (NARROW) t += wave;
        m0 = -64;
      };
      auto seek = [&] {  // to the first tile of the class at or after t, in this head or a later one
        for (;;) {
          while (t < t1) {
            if (REL) {
              if (tile_class(t) == CLASS) return;
              t += STEP;
              continue;
            }
            const int lt = t * QT / kTrainQTile;
            if (lt >= m0 + 64) {
              m0 = lt;
              mask = __ballot((lt + lane) * kTrainQTile < g.nq && limit_class(lt + lane) == CLASS);
            }
            const uint64_t rest = mask >> (lt - m0);
            if (rest & 1) return;
            if (NARROW) t += STEP;
            else t = (rest ? lt + __builtin_ctzll(rest) : m0 + 64) * (kTrainQTile / QT);
          }
          if (!MANY || ++hh >= h1) return;
          head();
        }
      };
      head();
      seek();
      if (MANY ? hh >= h1 : t >= t1) return;
      int h = hk * per + hh, now = t;
      fetch(h, now, 0);
      park_stat(masked_c, fetch_stat(h, now), now, 0);
      for (int b = 0;; b = BUFS == 2 ? b ^ 1 : 0) {
        if (NARROW) tile_ready();
        else tiles_ready();
        t += STEP;
        seek();
        const bool more = MANY ? hh < h1 : t < t1;
        if (MANY) h = hk * per + hh;
        float2_t st = {0.f, 0.f};
        if (more) {
          if (BUFS == 2) fetch(h, t, b ^ 1);
          st = fetch_stat(h, t);
        }
        if (k_wave < g.nk) tile(masked_c, now, b);
        if (!more) break;
        if (BUFS == 1) tile_read(), fetch(h, t, 0);
        park_stat(masked_c, st, t, BUFS == 2 ? b ^ 1 : 0);
        now = t;
      }
      if (!NARROW) __syncthreads();
    };
    // a bias changes with the head; without one the heads follow each other
    if (!REL && per > 1) {
      run(std::false_type{}, std::true_type{}, 0, per);
      run(std::true_type{}, std::true_type{}, 0, per);
    } else if (!REL) {
      run(std::false_type{}, std::false_type{}, 0, 1);
      run(std::true_type{}, std::false_type{}, 0, 1);
    }
    for (int hh = 0; REL && hh < per; ++hh) {
      if (i0 >= (hh + 1) * per_head || i1 <= hh * per_head) continue;
      const int h = hk * per + hh;
      // (wide: every wave is past the barrier that ended the head before, and the
      // first tile waits at one)
      if (NARROW) __syncthreads();
      stage_bias(tab, (const T*)a.rel, R, h, tid);
      if (NARROW) __syncthreads();
      far = bias_value((const T*)a.rel, R, h, R1);
      run(std::false_type{}, std::false_type{}, hh, hh + 1);
      run(std::true_type{}, std::false_type{}, hh, hh + 1);
    }
    if (V_LDS) tile_ready();  // (no tile may have waited for V)
    return again;
  };
  if (__syncthreads_or(pass(std::false_type{}))) (void)pass(std::true_type{});
  const int64_t first_row = g.k0 + k_first;
  char* const dk_out = a.dk.p + first_row * a.dk.row + hk * a.dk.head;
  char* const dv_out = a.dv.p + first_row * a.dv.row + hk * a.dv.head;
  float* const slot = parts == 1 ? nullptr
                                 : a.partial + ((size_t)g.slot_k + (size_t)((kblk * parts + part) * a.G + hk)) *
                                                   train_dkv_slot(ROWS, DH);
  if constexpr (NARROW) {
    __syncthreads();  // every wave has done its tiles
    Park<DH>::put(dk, bufs, lane);
    __syncthreads();
    add_parked<T, DH>(smem, 2 * BUFS * TB, slot, a.scale, dk_out, a.dk.row, g.nk - k_first, tid);
    __syncthreads();
    Park<DH>::put(dv, bufs, lane);
    __syncthreads();
    add_parked<T, DH>(smem, 2 * BUFS * TB, slot ? slot + ROWS * DH : nullptr, 1.f, dv_out, a.dv.row, g.nk - k_first,
                      tid);
    return;
  }
  if (slot) {
    const size_t r = wave * 32 + l32;
    if (exists) {
      store_partial<T, DH>(dk, slot + r * DH, hi);
      store_partial<T, DH>(dv, slot + (ROWS + r) * DH, hi);
    }
    return;
  }
  if (k_wave >= g.nk) return;
  lds_char* const stage = smem + wave * 32 * Gm::RB;
  store_rows<T, DH>(dk, a.scale, stage, dk_out + wave * 32 * a.dk.row, a.dk.row, g.nk - k_wave, lane);
  __builtin_amdgcn_wave_barrier();
  store_rows<T, DH>(dv, 1.f, stage, dv_out + wave * 32 * a.dv.row, a.dv.row, g.nk - k_wave, lane);
}

template <class T, int DH>
__global__ __launch_bounds__(256) void train_dkv_join_kernel(const TrainArgs a) {
  __shared__ __align__(16) char left_[256 * 16];
  lds_char* const left = (lds_char*)left_;
  const int unit = blockIdx.x / a.G, hk = blockIdx.x % a.G, tid = threadIdx.x;
  const TrainGroup g = a.groups[find_group<true>(a.groups, a.n_groups, unit, tid & 63)];
  const int parts = g.parts_k, local = unit - g.unit_k, ROWS = a.k_rows, kblk = local / parts,
            k_first = kblk * ROWS;
  if (parts == 1 || local % parts) return;
  const size_t slot = train_dkv_slot(ROWS, DH), step = (size_t)a.G * slot;
  const float* const p0 = a.partial + ((size_t)g.slot_k + (size_t)(kblk * parts * a.G + hk)) * slot;
  const int rows = min(ROWS, g.nk - k_first);
  const int64_t row = g.k0 + k_first;
  join_sums<T, DH>(p0, step, parts, rows, a.scale, a.dk.p + row * a.dk.row + hk * a.dk.head, a.dk.row, left, tid);
  join_sums<T, DH>(p0 + ROWS * DH, step, parts, rows, 1.f, a.dv.p + row * a.dv.row + hk * a.dv.head, a.dv.row,
                   left, tid);
}

template <class T, int DH, bool REL, bool NARROW>
hipError_t dkv_launch(const TrainArgs& a, hipStream_t s) {
  const size_t lds = dkv_lds_bytes<T, DH, NARROW>() + 4 * stat_floats<T, DH, NARROW>() +
                     (REL ? 4 * (size_t)bias_entries(a.R) : 0);
  static LdsAllowed so_far;
  const hipError_t e = allow_lds((const void*)train_dkv_kernel<T, DH, REL, NARROW>, lds, so_far);
  if (e != hipSuccess) return e;
  train_dkv_kernel<T, DH, REL, NARROW><<<place_grid(a.k_units, a.G, a.k_chunk), 256, lds, s>>>(a);
  return hipGetLastError();
}
template <class T, int DH>
hipError_t dkv_join(const TrainArgs& a, hipStream_t s) {
  train_dkv_join_kernel<T, DH><<<dim3((unsigned)a.k_units * a.G), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_train_dkv(bool bf, int dh, bool rel, const TrainArgs& a, hipStream_t s) {
  const bool narrow = a.k_narrow;
#define TX_CASE(T, D)                                                                                       \
  return narrow ? (rel ? dkv_launch<T, D, true, true>(a, s) : dkv_launch<T, D, false, true>(a, s))    \
                : (rel ? dkv_launch<T, D, true, false>(a, s) : dkv_launch<T, D, false, false>(a, s))
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

hipError_t launch_train_dkv_join(bool bf, int dh, const TrainArgs& a, hipStream_t s) {
  if (bf)
    return dh == 32 ? dkv_join<bf16, 32>(a, s) : dh == 64 ? dkv_join<bf16, 64>(a, s) : dkv_join<bf16, 128>(a, s);
  return dh == 32 ? dkv_join<float, 32>(a, s) : dh == 64 ? dkv_join<float, 64>(a, s) : dkv_join<float, 128>(a, s);
}

}  // namespace tx
