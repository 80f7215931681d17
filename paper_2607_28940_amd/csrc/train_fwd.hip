// Forward of the training attention (train_attn.h): O and lse of 128 queries of
// one (group, head) per block, in one pass over the visible keys with the
// running maximum and sum of the softmax.
#include "meta_put.h"
#include "train_attn.h"

#include <type_traits>

namespace tx {
namespace {

// Keys of a tile, tile buffers (K and V each) of a block or of a narrow block's
// wave, bytes of a tile, and bytes of all tiles.
template <class T, bool NARROW>
constexpr int key_tile() { return sizeof(T) == 2 && !NARROW ? 64 : 32; }
template <class T, int DH, bool NARROW>
constexpr int fwd_buffers() { return NARROW && sizeof(T) == 4 && DH == 128 ? 1 : 2; }
template <class T, int DH, bool NARROW>
constexpr int fwd_tile_bytes() { return key_tile<T, NARROW>() * Geo<T, DH>::RB; }
template <class T, int DH, bool NARROW>
constexpr int fwd_lds_bytes() {
  return (NARROW ? 4 : 1) * 2 * fwd_buffers<T, DH, NARROW>() * fwd_tile_bytes<T, DH, NARROW>();
}
// Wide blocks per CU: at d_head 64 and less four of 32 KB and 128 registers (98
// against 103 us for 17 k queries of 2.3 k keys at 64; three no better than two).
template <class T, int DH, bool NARROW>
constexpr int fwd_blocks() { return NARROW ? 1 : sizeof(T) == 2 && DH <= 64 ? 4 : 2; }

// Per wave and tile of KT keys: S^T = K Q^T with keys as rows, so a lane holds
// KT / 2 keys of one query and the softmax needs one exchange with lane l ^ 32;
// then O^T += V^T P^T, P^T taken from the accumulators as they are and V^T
// fragments read from the row-major tile (bf16: transposing LDS reads).
// K and V are double-buffered, one barrier per tile. P is rounded to bf16 for its
// product (2^-9 of a term), l sums what was not rounded.
// Measured, 8 heads: 147 k queries of 2.3 k keys at d_head 128 in 1.46 ms, 0.95
// PFLOP/s; 16384 causal tokens 0.53 ms, 1.04. At 128 the matrix units are busy 46%
// of the cycles, the vector units 43%, two waves a SIMD; at 64 a tile's 32
// exponentials and 150 other vector operations a lane bound it (4 x 8192 causal
// tokens 0.33 ms, 0.83 PFLOP/s).
template <class T, int DH, bool REL, bool NARROW>
__global__ __launch_bounds__(256, (fwd_blocks<T, DH, NARROW>())) void train_fwd_kernel(const TrainArgs a) {
  using Gm = Geo<T, DH>;
  using W = Wave<T, DH>;
  constexpr int KT = key_tile<T, NARROW>(), KB = KT / 32, TB = fwd_tile_bytes<T, DH, NARROW>();
  constexpr int BUFS = fwd_buffers<T, DH, NARROW>();
  extern __shared__ __align__(1024) char smem_[];
  lds_char* const smem = (lds_char*)smem_;
  lds_float* const tab = (lds_float*)(smem + fwd_lds_bytes<T, DH, NARROW>());
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
  // a group's last rows see the most keys (later events have longer prefixes): first
  const int qb = blocks - 1 - local / parts;
  const int q_first = qb * ROWS;
  const int hk = h0 / (a.H / a.G);

  // keys that any row of the block sees, and the block's share of them
  int k_end;
  if (REL) {
    k_end = min(g.nq, q_first + ROWS);
  } else {
    const TileLim* tl = a.tile_lim + g.qt0 + q_first / kTrainQTile;
    k_end = tl[0].hi;
    if (ROWS > kTrainQTile && q_first + kTrainQTile < g.nq) k_end = max(k_end, tl[1].hi);
  }
  const int R = REL ? a.R : 0, R1 = max(R, 1) - 1;  // R1: the first distance of the last bucket
  if (REL) stage_bias(tab, (const T*)a.rel, R, h, tid);
  const float far = REL ? bias_value((const T*)a.rel, R, h, R1) : 0.f;
  int t_begin = 0;
  // a last bucket that masks leaves a window of the R - 1 nearest keys
  if (REL && far == -INFINITY) t_begin = max(0, q_first - (R - 2)) / KT;
  int t_end = (k_end + KT - 1) / KT;
  // Tiles before t_plain are visible to every row of the block, with one bias
  // for all pairs; a large one goes to each logit, as there is no telling how
  // it rounds them.
  int t_plain;
  if (REL) {
    t_plain = fabsf(far) < 0x1p20f ? max(0, q_first - R1 + 1) / KT : 0;
  } else {
    const TileLim* tl = a.tile_lim + g.qt0 + q_first / kTrainQTile;
    t_plain = tl[0].lo;
    if (ROWS > kTrainQTile && q_first + kTrainQTile < g.nq) t_plain = min(t_plain, tl[1].lo);
    t_plain /= KT;
  }
  if (parts > 1) {
    const int n = max(0, t_end - t_begin);
    t_end = t_begin + (int)((int64_t)n * (part + 1) / parts);
    t_begin += (int)((int64_t)n * part / parts);
  }
  t_plain = min(t_plain, t_end);

  const int q_wave = q_first + w_row;  // first query of the wave, within the group
  const int q_row = q_wave + l32;
  const bool exists = q_row < g.nq;
  int lim = 0;  // visible keys of the lane's query
  if (exists) lim = REL ? q_row + 1 : a.row_lim[g.q0 + q_row - a.q_base];
  int lim_hi = 0;  // the largest of the wave's rows
  if (REL) {
    if (q_wave < g.nq) lim_hi = min(q_wave + 32, g.nq);
  } else {
    int up = lim;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) up = max(up, __shfl_xor(up, m));
    lim_hi = uniform(up);
  }

  floatx16 o[Gm::NB];
  float m, l;

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
  // One pass over the keys. A masked tile whose values are not all finite has
  // to keep them from the pairs out of sight; that is rare, and its code would
  // cost every other tile registers, so such a block starts again with STRICT
  // (same results but for the sums that those values reach).
  auto pass = [&](auto strict_c) {
    constexpr bool STRICT = decltype(strict_c)::value;
    u32x4_t qf[Gm::NC];
    load_row_frags<T, DH>(a.q.p + (int64_t)(g.q0 + q_row) * a.q.row + h * a.q.head, exists, hi, qf);
    m = -INFINITY, l = 0.f;
#pragma unroll
    for (int db = 0; db < Gm::NB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
    bool again = false;
    // With three or four waves on a SIMD a wave's products go before the others'
    // softmax, so that the matrix unit is not kept waiting (8192 causal tokens, 4
    // sequences of 8 heads at d_head 64: 340 against 356 us; two waves at 128: 1.49
    // against 1.47 ms for 147 k queries of 2.3 k keys, left alone).
    constexpr bool FIRST = fwd_blocks<T, DH, NARROW>() > 2;
    // One tile for one wave; MASKED: pairs may be out of sight or near enough for
    // a bias of their own.
    auto tile = [&](auto masked_c, int t, int b) {
      constexpr bool MASKED = decltype(masked_c)::value;
      const int k0 = t * KT;
      const lds_char* const sK = bufs + b * TB;
      const lds_char* const sV = bufs + (BUFS + b) * TB;
      floatx16 s[KB];
      if (FIRST) __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) w.rows_product(sK, kb, qf, s[kb]);
      if (FIRST) __builtin_amdgcn_s_setprio(0);
      // logits as fma(s, mul, add): plain tiles scale here, masked ones were
      // brought to base-2 logits already
      const float mul = MASKED ? 1.f : a.scale_log2, add = MASKED ? 0.f : far;
      // table entry of the pair with the tile's key 4 hi (distances past the
      // padding are all in the last bucket)
      const int d0 = min(q_row - k0, R1 + kBiasPad - 1) - 4 * hi + kBiasPad;
      if (MASKED) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int key = kb * 32 + 8 * (v >> 2) + (v & 3);
            if (REL) {
              const float bias = tab[d0 - key];
              s[kb][v] = bias == -INFINITY ? -INFINITY : fmaf(s[kb][v], a.scale_log2, bias);
            } else {
              s[kb][v] = key < lim - k0 - 4 * hi ? s[kb][v] * a.scale_log2 : -INFINITY;
            }
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kb][v]);
      mx = fmaf(xor32_max(mx), mul, add);
      // The reference m moves only when this tile would push a probability above
      // 2^8 (fine for fp32 sums and for bf16 P, whose rounding is relative); O / l
      // does not depend on which reference was used.
      const bool bump = mx > m + 8.f;
      if (__any(bump)) {
        const float m_new = bump ? mx : m;
        const float alpha = bump ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < Gm::NB; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
        m = m_new;
      }
      const float off = m == -INFINITY ? 0.f : add - m;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          s[kb][v] = __builtin_amdgcn_exp2f(fmaf(s[kb][v], mul, off));
          l += s[kb][v];
        }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if (MASKED && !STRICT) again |= w.rows_not_finite(sV, kb);
        if constexpr (MASKED && STRICT) {
          uint32_t vis = 0;
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int key = kb * 32 + 8 * (v >> 2) + (v & 3);
            const bool see = REL ? tab[d0 - key] != -INFINITY : key < lim - k0 - 4 * hi;
            vis |= see ? 1u << v : 0u;
          }
          w.cols_mma_strict(sV, kb, s[kb], vis, o);
        } else {
          if (FIRST) __builtin_amdgcn_s_setprio(1);
          w.cols_mma(sV, kb, s[kb], o);
          if (FIRST) __builtin_amdgcn_s_setprio(0);
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
    if (NARROW) __syncthreads();  // (the bias table)
    if (t < t_end) fetch(t, 0);
    pin(qf), pin(lim);
    ready();
    run(std::false_type{}, t_plain, q_wave < g.nq);
    run(std::true_type{}, t_end, true);
    if (NARROW) __syncthreads();
    return again;
  };
  if (__syncthreads_or(pass(std::false_type{}))) (void)pass(std::true_type{});
  l = xor32_sum(l);
  const int64_t first_row = g.q0 + q_first;
  char* const out = a.o.p + first_row * a.o.row + h * a.o.head;
  float* const slot = parts == 1 ? nullptr
                                 : a.partial + ((size_t)g.slot_q + (size_t)((qb * parts + part) * a.H + h)) *
                                                   train_fwd_slot(ROWS, DH);
  if constexpr (NARROW) {
    // (the pass ended on a barrier: the tiles are free)
    constexpr int STEP = 2 * BUFS * TB;
    lds_float* const ml = (lds_float*)(bufs + Park<DH>::BYTES);
    Park<DH>::put(o, bufs, lane);
    if (hi == 0) ml[l32] = m, ml[32 + l32] = l;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) {
      const int r = (tid + 256 * i) / Park<DH>::UNITS, u = (tid + 256 * i) % Park<DH>::UNITS;
      if (q_first + r >= g.nq) continue;
      float mw[4], lw[4], top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int wv = 0; wv < 4; ++wv) {
        const lds_float* const x = (const lds_float*)(smem + wv * STEP + Park<DH>::BYTES);
        mw[wv] = x[r], lw[wv] = x[32 + r];
        top = fmaxf(top, mw[wv]);
      }
      floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int wv = 0; wv < 4; ++wv) {
        const float wgt = mw[wv] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw[wv] - top);  // (as in the join)
        const floatx4 x = *Park<DH>::at(smem + wv * STEP, r, u);
        sum += wgt * lw[wv];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] += wgt * x[t];
      }
      if (slot) {
        *reinterpret_cast<floatx4*>(slot + r * DH + 4 * u) = acc;
        if (u == 0) slot[ROWS * DH + r] = top, slot[ROWS * (DH + 1) + r] = sum;
      } else {
        store4((T*)(out + r * a.o.row) + 4 * u, acc, sum == 0.f ? 0.f : 1.f / sum);
        if (u == 0)
          a.lse[(int64_t)h * a.lse_ld + first_row + r] =
              sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kTrainLn2;
      }
    }
    return;
  }
  if (slot) {
    const int r = w_row + l32;
    if (exists) {
      store_partial<T, DH>(o, slot + (size_t)r * DH, hi);
      if (hi == 0) slot[ROWS * DH + r] = m, slot[ROWS * (DH + 1) + r] = l;
    }
    return;
  }
  // l is 0 only for a row without a visible key: its output is 0, its lse minus infinity
  const int n_rows = g.nq - q_wave;
  if (exists && hi == 0)
    a.lse[(int64_t)h * a.lse_ld + g.q0 + q_row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kTrainLn2;
  if (n_rows > 0)
    store_rows<T, DH>(o, l == 0.f ? 0.f : 1.f / l, smem + wave * 32 * Gm::RB, out + w_row * a.o.row, a.o.row, n_rows,
                      lane);
}

// Joins the parts of a divided block of queries: with the parts' maxima m_p and
// sums l_p, O = sum_p w_p O_p / sum_p w_p l_p, w_p = 2^(m_p - max m).
template <class T, int DH>
__global__ __launch_bounds__(256) void train_fwd_join_kernel(const TrainArgs a) {
  __shared__ __align__(16) char left_[256 * 20];
  lds_char* const smem = (lds_char*)left_;
  const int unit = blockIdx.x / a.H, h = blockIdx.x % a.H, tid = threadIdx.x;
  const TrainGroup g = a.groups[find_group<false>(a.groups, a.n_groups, unit, tid & 63)];
  const int parts = g.parts_q, local = unit - g.unit_q, qb = local / parts;
  if (parts == 1 || local % parts) return;
  const int ROWS = a.q_rows, rows = min(ROWS, g.nq - qb * ROWS);
  const size_t SLOT = train_fwd_slot(ROWS, DH);
  const float* const p0 = a.partial + ((size_t)g.slot_q + (size_t)(qb * parts * a.H + h)) * SLOT;
  const size_t step = SLOT * a.H;
  const Joiner<DH> j(rows, tid);
  lds_floatx4* const left = (lds_floatx4*)smem;
  lds_float* const left_l = (lds_float*)(smem + 256 * 16);
  for (int r0 = 0; r0 < rows; r0 += j.at_once) {
    const int r = r0 + j.slot;
    float top = -INFINITY, l = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    if (r < rows) {
#pragma unroll 8
      for (int p = 0; p < parts; ++p) top = fmaxf(top, p0[p * step + ROWS * DH + r]);
#pragma unroll 4
      for (int p = j.share; p < parts; p += j.shares) {
        const float* const s = p0 + p * step;
        const float m = s[ROWS * DH + r], lp = s[ROWS * (DH + 1) + r];
        const floatx4 x = *reinterpret_cast<const floatx4*>(s + (size_t)r * DH + j.f);
        // a part without a visible key holds zeros and m = -inf (l says whether it is one: a
        // part of nothing but NaN logits has that m too)
        const float wgt = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
        l += wgt * lp;
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] += wgt * x[t];
      }
    }
    if (j.shares > 1) {
      left[tid] = acc;
      left_l[tid] = l;
      __syncthreads();
      for (int q = 1; q < j.shares && j.share == 0; ++q) {
        const int from = tid + q * j.at_once * Joiner<DH>::LPR;
        const floatx4 x = left[from];
        l += left_l[from];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] += x[t];
      }
      __syncthreads();
    }
    if (r >= rows || j.share) continue;
    const int64_t row = g.q0 + qb * ROWS + r;
    if (j.f == 0)
      a.lse[(int64_t)h * a.lse_ld + row] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kTrainLn2;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    store4((T*)(a.o.p + row * a.o.row + h * a.o.head) + j.f, acc, inv);
  }
}

// The event form's key limits: a wave per 64-row query tile finds each row's
// event (the last whose first row is not past it: events may be empty) and keeps
// its prefix, with the tile's smallest and largest.
__device__ __forceinline__ void key_limits(const TrainGroup* groups, int n_groups, const int32_t* ev_row,
                                           const int32_t* ev_prefix, int32_t* __restrict__ row_lim, int q_base,
                                           TileLim* __restrict__ tile_lim) {
  const int lane = threadIdx.x, tile = blockIdx.x;
  // the last group whose first tile is not past this one
  int lo = 0, n = n_groups;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    const bool ok = i < n && groups[lo + i].qt0 <= tile;
    const int c = max(1, (int)__popcll(__ballot(ok)));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  const TrainGroup g = groups[uniform(lo)];
  const int r = (tile - g.qt0) * kTrainQTile + lane;
  const bool exists = r < g.nq;
  int lim = 0;
  if (exists) {
    const int row = g.q0 + r;
    int a = g.e0, b = g.e1 - 1;  // last event in a .. b whose first row is <= row
    while (a < b) {
      const int mid = (a + b + 1) >> 1;
      if (ev_row[mid] <= row) a = mid;
      else b = mid - 1;
    }
    lim = ev_prefix[a];
    row_lim[row - q_base] = lim;
  }
  int mn = exists ? lim : 0x7fffffff, mx = lim;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    mn = min(mn, __shfl_xor(mn, m));
    mx = max(mx, __shfl_xor(mx, m));
  }
  if (lane == 0) tile_lim[tile] = TileLim{mn, mx};
}

__global__ __launch_bounds__(64) void train_limits_kernel(const TrainGroup* __restrict__ groups, int n_groups,
                                                         const int32_t* __restrict__ ev_row,
                                                         const int32_t* __restrict__ ev_prefix, int32_t* row_lim,
                                                         int q_base, TileLim* tile_lim) {
  key_limits(groups, n_groups, ev_row, ev_prefix, row_lim, q_base, tile_lim);
}

// The same from metadata that comes as arguments, which the launch also writes
// to where the next ones read it: one launch instead of two.
__global__ __launch_bounds__(64) void train_put_limits_kernel(uint32_t* __restrict__ dst, int words, int n_groups,
                                                             int o_row, int o_prefix, int32_t* row_lim, int q_base,
                                                             TileLim* tile_lim, const MetaArg m) {
  for (int i = blockIdx.x * 64 + threadIdx.x; i < words; i += gridDim.x * 64) dst[i] = m.w[i];
  const char* const src = (const char*)m.w;
  key_limits((const TrainGroup*)src, n_groups, (const int32_t*)(src + o_row), (const int32_t*)(src + o_prefix), row_lim,
             q_base, tile_lim);
}

template <class T, int DH, bool REL, bool NARROW>
hipError_t fwd(const TrainArgs& a, hipStream_t s) {
  const size_t lds = fwd_lds_bytes<T, DH, NARROW>() + (REL ? 4 * (size_t)bias_entries(a.R) : 0);
  static LdsAllowed so_far;
  const hipError_t e = allow_lds((const void*)train_fwd_kernel<T, DH, REL, NARROW>, lds, so_far);
  if (e != hipSuccess) return e;
  train_fwd_kernel<T, DH, REL, NARROW><<<place_grid(a.n_units, a.H >> a.pack, a.q_chunk), 256, lds, s>>>(a);
  return hipGetLastError();
}

template <class T, int DH>
hipError_t fwd_join(const TrainArgs& a, hipStream_t s) {
  train_fwd_join_kernel<T, DH><<<dim3((unsigned)a.n_units * a.H), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_train_fwd(bool bf, int dh, bool rel, const TrainArgs& a, hipStream_t s) {
  const bool narrow = a.q_narrow;
#define TX_CASE(T, D)                                                                   \
  return narrow ? (rel ? fwd<T, D, true, true>(a, s) : fwd<T, D, false, true>(a, s))    \
                : (rel ? fwd<T, D, true, false>(a, s) : fwd<T, D, false, false>(a, s))
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

hipError_t launch_train_fwd_join(bool bf, int dh, const TrainArgs& a, hipStream_t s) {
  if (bf)
    return dh == 32 ? fwd_join<bf16, 32>(a, s) : dh == 64 ? fwd_join<bf16, 64>(a, s) : fwd_join<bf16, 128>(a, s);
  return dh == 32 ? fwd_join<float, 32>(a, s) : dh == 64 ? fwd_join<float, 64>(a, s) : fwd_join<float, 128>(a, s);
}

hipError_t launch_train_limits(const TrainGroup* groups, int32_t n_groups, int32_t n_tiles, const int32_t* ev_row,
                               const int32_t* ev_prefix, int32_t* row_lim, int32_t q_base, TileLim* tile_lim,
                               hipStream_t s) {
  train_limits_kernel<<<n_tiles, 64, 0, s>>>(groups, n_groups, ev_row, ev_prefix, row_lim, q_base, tile_lim);
  return hipGetLastError();
}

hipError_t launch_train_put_limits(void* dst, const void* meta, size_t bytes, int32_t n_groups, int32_t n_tiles,
                                   size_t o_row, size_t o_prefix, int32_t* row_lim, int32_t q_base, TileLim* tile_lim,
                                   hipStream_t s) {
  MetaArg m;
  memcpy(m.w, meta, bytes);
  const int words = (int)((bytes + 3) / 4);
  if (bytes % 4) memset((char*)m.w + bytes, 0, 4 - bytes % 4);
  train_put_limits_kernel<<<n_tiles, 64, 0, s>>>((uint32_t*)dst, words, n_groups, (int)o_row, (int)o_prefix, row_lim,
                                                 q_base, tile_lim, m);
  return hipGetLastError();
}

}  // namespace tx
