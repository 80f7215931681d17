// Backward of the training attention (train_attn.h), key side: dk and dv of 128
// keys of one (group, key head) per block, summed over the queries of every
// query head that reads the key head. Keys that no query sees get zeros.
#include "train_attn.h"

namespace tx {
namespace {

template <class T>
constexpr int query_tile() { return sizeof(T) == 2 ? 64 : 32; }

template <class T, int DH>
constexpr int dkv_tile_bytes() { return query_tile<T>() * Geo<T, DH>::RB; }

// A wave owns 32 keys, whose K and V fragments stay in registers. Per 32
// queries: S = Q K^T and dP = dO V^T (lanes = keys), P and dS = P (dP - D),
// then dV^T += dO^T P and dK^T += Q^T dS with P and dS taken from the
// accumulators and the columns of the dO and Q tiles read from LDS (bf16:
// transposing reads). P and dS are rounded to bf16 for those products. Q, dO
// and the rows' lse, D and key limits are double-buffered, one barrier a tile.
template <class T, int DH, bool REL>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void train_dkv_kernel(const TrainArgs a) {
  using Gm = Geo<T, DH>;
  using W = Wave<T, DH>;
  constexpr int QT = query_tile<T>(), QB = QT / 32, TB = dkv_tile_bytes<T, DH>();
  extern __shared__ __align__(1024) char smem_[];
  lds_char* const smem = (lds_char*)smem_;
  lds_float* const stat = (lds_float*)(smem + 4 * TB);  // [2 buffers][lse2, D, limits][QT]
  lds_float* const tab = stat + 6 * QT;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int unit = blockIdx.x / a.G, hk = blockIdx.x % a.G, per = a.H / a.G;
  const TrainGroup g = a.groups[find_group<true>(a.groups, a.n_groups, unit, lane)];
  const int parts = g.parts_k, local = unit - g.unit_k, part = local % parts, kblk = local / parts;
  const int k_first = kblk * kTrainRows, k_wave = k_first + wave * 32, key = k_wave + l32;
  const bool exists = key < g.nk;
  const int R = REL ? a.R : 0;

  u32x4_t kf[Gm::NC], vf[Gm::NC];
  load_row_frags<T, DH>(a.k.p + (int64_t)(g.k0 + key) * a.k.row + hk * a.k.head, exists, hi, kf);
  load_row_frags<T, DH>(a.v.p + (int64_t)(g.k0 + key) * a.v.row + hk * a.v.head, exists, hi, vf);

  floatx16 dk[Gm::NB], dv[Gm::NB];
#pragma unroll
  for (int db = 0; db < Gm::NB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[db][v] = 0.f, dv[db][v] = 0.f;

  // Work list of the block: (query head, query tile), heads outermost. Causal
  // rows before the block's first key do not see it; with a last bucket that
  // masks (window), rows more than R - 2 past its last key do not either
  // (their tiles are masked one by one below, per head).
  const int nqt = (g.nq + QT - 1) / QT, t0 = REL ? min(nqt, k_first / QT) : 0, per_head = nqt - t0;
  int i0 = 0, i1 = per * per_head;
  if (parts > 1) {
    const int n = i1;
    i1 = (int)((int64_t)n * (part + 1) / parts);
    i0 = (int)((int64_t)n * part / parts);
  }
  // next item at or after i whose tile sees the block's keys
  auto next = [&](int i) {
    if (!REL) {
      for (; i < i1; ++i) {
        const int t = t0 + i % per_head;
        // QT = 64: one limit tile per query tile; QT = 32: two query tiles per limit tile
        if (a.tile_lim[g.qt0 + t * QT / kTrainQTile].hi > k_first) break;
      }
    }
    return i;
  };
  const W w(lane);
  const TileDma<T, DH, QT> qd(wave, lane, a.q.row), dd(wave, lane, a.dO.row);
  // The rows' statistics: threads 0 .. QT - 1 lse, then D, then limits; fetched
  // with the tile, parked in LDS once the tile before has been computed.
  auto fetch_stat = [&](int i) {
    const int h = hk * per + i / per_head, r = (t0 + i % per_head) * QT + tid % QT, kind = tid / QT;
    const bool ok = r < g.nq;
    float x = 0.f;
    if (kind == 0) {
      x = ok ? a.lse[(int64_t)h * a.lse_ld + g.q0 + r] : -INFINITY;
      x = x == -INFINITY ? INFINITY : x * kTrainLog2e;  // probabilities 0 for rows that see nothing
    } else if (kind == 1) {
      x = ok ? a.D[(int64_t)h * a.D_ld + g.q0 + r - a.q_base] : 0.f;
    } else if (kind == 2 && !REL) {
      x = __int_as_float(ok ? a.row_lim[g.q0 + r - a.q_base] : 0);
    }
    return x;
  };
  auto park_stat = [&](float x, int b) {
    if (tid < 3 * QT) stat[b * 3 * QT + tid] = x;
  };
  auto fetch = [&](int i, int b) {
    const int h = hk * per + i / per_head, r = (t0 + i % per_head) * QT;
    qd.load(a.q.p + (int64_t)(g.q0 + r) * a.q.row + h * a.q.head, g.nq - r, smem + b * TB);
    dd.load(a.dO.p + (int64_t)(g.q0 + r) * a.dO.row + h * a.dO.head, g.nq - r, smem + (2 + b) * TB);
  };
  int i = next(i0), b = 0, h_tab = -1;
  float far = 0.f;
  if (i < i1) {
    fetch(i, 0);
    park_stat(fetch_stat(i), 0);
  }
  while (i < i1) {
    const int h = hk * per + i / per_head;
    if (REL && h != h_tab) {
      // (every wave is past the barrier that ended the last tile of the head before)
      stage_bias(tab, (const T*)a.rel, R, h, tid);
      far = bias_value((const T*)a.rel, R, h, max(R, 1) - 1);
      h_tab = h;
    }
    __syncthreads();
    const int in = next(i + 1);
    float st = 0.f;
    if (in < i1) {
      fetch(in, b ^ 1);
      st = fetch_stat(in);
    }
    const lds_char* const sQ = smem + b * TB;
    const lds_char* const sO = smem + (2 + b) * TB;
    const lds_float* const ss = stat + b * 3 * QT;
    const int q0 = (t0 + i % per_head) * QT;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int qr = q0 + 32 * qb;  // first query of the 32
      if (qr >= g.nq || k_wave >= g.nk) continue;
      if (REL && qr + 31 < k_wave) continue;
      const bool near = REL && (qr - (k_wave + 31) < R - 1 || fabsf(far) >= 0x1p20f);
      if (REL && far == -INFINITY && qr - (k_wave + 31) >= R - 1) continue;
      floatx16 s, p;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = 0.f, p[v] = 0.f;
#pragma unroll
      for (int c = 0; c < Gm::NC; ++c) s = W::rows_mma(w.row_frag(sQ, qb, c), kf[c], s);
#pragma unroll
      for (int c = 0; c < Gm::NC; ++c) p = W::rows_mma(w.row_frag(sO, qb, c), vf[c], p);
      const int d0 = min(qr - key, R - 1 + kBiasPad - 32) + 4 * hi + kBiasPad;
      bool masked = near;
      uint32_t vis = 0xffff;
      if (!REL) {
        bool some = false;
        vis = 0;
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
          const floatx4 lm = *reinterpret_cast<const lds_floatx4*>(ss + 2 * QT + 32 * qb + 8 * gq + 4 * hi);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const bool see = key < __float_as_int(lm[t]);
            vis |= see ? 1u << (4 * gq + t) : 0u;
            some |= !see;
          }
        }
        masked = __any(some);
      }
#pragma unroll
      for (int gq = 0; gq < 4; ++gq) {
        const floatx4 ls = *reinterpret_cast<const lds_floatx4*>(ss + 32 * qb + 8 * gq + 4 * hi);
        const floatx4 Dv = *reinterpret_cast<const lds_floatx4*>(ss + QT + 32 * qb + 8 * gq + 4 * hi);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int v = 4 * gq + t;
          float e;
          if (masked) {
            const float bias = REL ? tab[d0 + 8 * gq + t] : 0.f;
            if (REL && bias == -INFINITY) vis &= ~(1u << v);
            const float lg = fmaf(s[v], a.scale_log2, bias);
            e = (vis >> v) & 1 ? __builtin_amdgcn_exp2f(lg - ls[t]) : 0.f;
            p[v] = (vis >> v) & 1 ? e * (p[v] - Dv[t]) : 0.f;
          } else {
            e = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, far - ls[t]));
            p[v] = e * (p[v] - Dv[t]);
          }
          s[v] = e;
        }
      }
      if (masked && w.rows_not_finite(sO, qb)) w.cols_mma_strict(sO, qb, s, vis, dv);
      else w.cols_mma(sO, qb, s, dv);
      if (masked && w.rows_not_finite(sQ, qb)) w.cols_mma_strict(sQ, qb, p, vis, dk);
      else w.cols_mma(sQ, qb, p, dk);
    }
    if (in < i1) park_stat(st, b ^ 1);
    i = in;
    b ^= 1;
    if (REL && i < i1 && hk * per + i / per_head != h_tab) __syncthreads();  // the table changes: all waves are done with it
  }
  __syncthreads();  // the tiles are free
  if (parts > 1) {
    float* const slot =
        a.partial + ((size_t)g.slot_k + (size_t)((kblk * parts + part) * a.G + hk)) * (2 * kTrainRows * DH);
    const size_t r = wave * 32 + l32;
    store_partial<T, DH>(dk, slot + r * DH, hi);
    store_partial<T, DH>(dv, slot + (kTrainRows + r) * DH, hi);
    return;
  }
  if (k_wave >= g.nk) return;
  const int64_t row = g.k0 + k_wave;
  lds_char* const stage = smem + wave * 32 * Gm::RB;
  store_rows<T, DH>(dk, a.scale, stage, a.dk.p + row * a.dk.row + hk * a.dk.head, a.dk.row, g.nk - k_wave, lane);
  __builtin_amdgcn_wave_barrier();
  store_rows<T, DH>(dv, 1.f, stage, a.dv.p + row * a.dv.row + hk * a.dv.head, a.dv.row, g.nk - k_wave, lane);
}

template <class T, int DH>
__global__ __launch_bounds__(256) void train_dkv_merge_kernel(const TrainArgs a) {
  const int unit = blockIdx.x / a.G, hk = blockIdx.x % a.G, tid = threadIdx.x;
  const TrainGroup g = a.groups[find_group<true>(a.groups, a.n_groups, unit, tid & 63)];
  const int parts = g.parts_k, local = unit - g.unit_k;
  if (parts == 1 || local % parts) return;
  const int kblk = local / parts, rows = min(kTrainRows, g.nk - kblk * kTrainRows);
  constexpr size_t SLOT = (size_t)2 * kTrainRows * DH;
  const float* const p0 = a.partial + ((size_t)g.slot_k + (size_t)(kblk * parts * a.G + hk)) * SLOT;
  constexpr int LPR = DH / 4;
  for (int i = tid; i < 2 * rows * LPR; i += 256) {
    const int which = i / (rows * LPR), j = i % (rows * LPR), r = j / LPR, f = j % LPR * 4;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) {
      const floatx4 x =
          *reinterpret_cast<const floatx4*>(p0 + p * SLOT * a.G + (size_t)(which * kTrainRows + r) * DH + f);
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] += x[t];
    }
    const HeadRows& d = which ? a.dv : a.dk;
    const float mul = which ? 1.f : a.scale;
    T* const out = (T*)(d.p + (int64_t)(g.k0 + kblk * kTrainRows + r) * d.row + hk * d.head) + f;
#pragma unroll
    for (int t = 0; t < 4; ++t) out[t] = (T)(acc[t] * mul);
  }
}

template <class T, int DH, bool REL>
hipError_t dkv_launch(const TrainArgs& a, int32_t n_units, hipStream_t s) {
  const size_t lds = 4 * dkv_tile_bytes<T, DH>() + 6 * 4 * query_tile<T>() + (REL ? 4 * (size_t)bias_entries(a.R) : 0);
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void*)train_dkv_kernel<T, DH, REL>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  train_dkv_kernel<T, DH, REL><<<dim3((unsigned)n_units * a.G), 256, lds, s>>>(a);
  return hipGetLastError();
}
template <class T, int DH>
hipError_t dkv_merge(const TrainArgs& a, int32_t n_units, hipStream_t s) {
  train_dkv_merge_kernel<T, DH><<<dim3((unsigned)n_units * a.G), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_train_dkv(bool bf, int dh, bool rel, const TrainArgs& a, int32_t n, hipStream_t s) {
#define TX_CASE(T, D) return rel ? dkv_launch<T, D, true>(a, n, s) : dkv_launch<T, D, false>(a, n, s)
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

hipError_t launch_train_dkv_merge(bool bf, int dh, const TrainArgs& a, int32_t n, hipStream_t s) {
  if (bf)
    return dh == 32 ? dkv_merge<bf16, 32>(a, n, s) : dh == 64 ? dkv_merge<bf16, 64>(a, n, s) : dkv_merge<bf16, 128>(a, n, s);
  return dh == 32 ? dkv_merge<float, 32>(a, n, s) : dh == 64 ? dkv_merge<float, 64>(a, n, s) : dkv_merge<float, 128>(a, n, s);
}

}  // namespace tx
