// Preference loss over the action head's logits: paired log ratios.
//
// For row r with logits z and observed action c: log p_r = z_c - lse, lse = log
// sum_j exp z_j. An answer's log p is the sum over its rows; a pair's margin is
// m = beta ((log p_w - ref_w) - (log p_l - ref_l)) and its loss
//   -(1 - eps) log sigmoid(m) - eps log sigmoid(-m),
// whose derivative by m is sigmoid(m) - (1 - eps). So a row's gradient is
//   dz = coef (onehot_c - softmax z),  coef = +- dloss beta (sigmoid(m) - (1 - eps)).
// The margin needs every row of both answers before any gradient exists, so the
// logits are read twice: once for lse (kept per row) and log p, once for dz.
// Both passes are bound by that traffic: 6589 rows of 32003 bf16 logits (422 MB)
// take 105 us to read (75 once nothing is left to write back) and 157 us for their
// gradient, 4.8 TB/s together.
#include "preference.h"
#include "wave_reduce.h"

namespace tx {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float to_f(bf16 x) { return (float)x; }
__device__ __forceinline__ float to_f(float x) { return x; }

__global__ __launch_bounds__(256) void pref_offsets_kernel(int32_t* __restrict__ dst, const PrefOffsets a) {
  // thread t sums lengths t * per .. , the block scans the threads' sums
  constexpr int per = PrefOffsets::kLengths / 256;
  __shared__ int32_t sums[4];
  const int tid = threadIdx.x, lane = tid & 63;
  int32_t len[per], own = 0;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const int k = tid * per + i;
    len[i] = k < a.n ? a.len[k] : 0;
    own += len[i];
  }
  int32_t up_to = own;  // inclusive over the wave
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t x = __shfl_up(up_to, d);
    if (lane >= d) up_to += x;
  }
  if (lane == 63) sums[tid >> 6] = up_to;
  __syncthreads();
  int32_t at = a.base + up_to - own;
  for (int w = 0; w < (tid >> 6); ++w) at += sums[w];
  if (tid == 0) dst[0] = a.base;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    at += len[i];
    if (tid * per + i < a.n) dst[tid * per + i + 1] = at;
  }
}

// (max, sum of exp(x - max)) of two disjoint sets; empty: (-inf, 0).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float ref = top == -INFINITY ? 0.f : top;
  s = s * __builtin_amdgcn_exp2f((m - ref) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - ref) * kLog2e);
  m = top;
}

// 16 bytes of a row as floats
template <class T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  T x[N];
};
template <class T>
__device__ __forceinline__ Vec<T> load_vec(const T* p) {
  return __builtin_bit_cast(Vec<T>, *reinterpret_cast<const u32x4_t*>(p));
}

// Elements of a row before its first 16-byte boundary.
template <class T>
__device__ __forceinline__ int head_of(const T* row, int k) {
  return min(k, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
}

// An answer may have a thousand rows of a few nats each, of whose sum the margin
// keeps a small difference: log p of a row is taken and summed in 64 bits, so that
// only the roundings inside s (2^-24 of a row's terms) reach the loss.
__device__ __forceinline__ void finish_row(float m, float s, float z_act, bool counts, float* lse, double* picked) {
  const bool some = m != -INFINITY;
  const double l = some ? (double)m + log((double)s) : 0.0;
  *lse = some ? (float)l : -INFINITY;
  *picked = counts && some ? (double)z_act - l : 0.0;
}

// k <= 64: W lanes (a power of two >= k) hold a row, one element each.
template <class T>
__global__ __launch_bounds__(256) void pref_rows_narrow(const T* __restrict__ z, int64_t ld, int k, int W,
                                                       const int32_t* __restrict__ act, int64_t row0, int64_t n,
                                                       float* __restrict__ row_lse, double* __restrict__ picked) {
  const int j = threadIdx.x & (W - 1);
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / W;
  const bool ok = i < n;
  const int a = ok ? act[row0 + i] : -1;
  const float x = ok && j < k ? to_f(z[(row0 + i) * ld + j]) : -INFINITY;
  float m = x;
  for (int d = 1; d < W; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  float s = m == -INFINITY ? 0.f : expf(x - m);
  float za = j == a ? x : 0.f;
  for (int d = 1; d < W; d <<= 1) s += __shfl_xor(s, d), za += __shfl_xor(za, d);
  // (a not finite logit elsewhere stays out of za; the action's own stays in)
  if (ok && j == 0) finish_row(m, s, za, a >= 0 && a < k, row_lse + row0 + i, picked + i);
}

// The scalar head: logits [0, s], lse = log(1 + exp s), action 1 picks s.
template <class T>
__global__ __launch_bounds__(256) void pref_rows_scalar(const T* __restrict__ z, int64_t ld,
                                                       const int32_t* __restrict__ act, int64_t row0, int64_t n,
                                                       float* __restrict__ row_lse, double* __restrict__ picked) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int a = act[row0 + i];
  const float s = to_f(z[(row0 + i) * ld]);
  // log(1 + exp s) = max(s, 0) + log1p(exp(-|s|)); log p of the action directly,
  // so that a sure answer keeps its digits
  const float tail = log1pf(expf(-fabsf(s)));
  row_lse[row0 + i] = fmaxf(s, 0.f) + tail;
  picked[i] = a == 1 ? -((double)fmaxf(-s, 0.f) + tail) : a == 0 ? -((double)fmaxf(s, 0.f) + tail) : 0.0;
}

// Wider rows: a block of 256 per row, 16 bytes a lane between the row's ragged
// ends, each thread its own running maximum and sum.
template <class T>
__global__ __launch_bounds__(256) void pref_rows_wide(const T* __restrict__ z, int64_t ld, int k,
                                                     const int32_t* __restrict__ act, int64_t row0,
                                                     float* __restrict__ row_lse, double* __restrict__ picked) {
  __shared__ float sm[4], ss[4];
  constexpr int N = Vec<T>::N;
  const int tid = threadIdx.x;
  const int64_t i = blockIdx.x, row = row0 + i;
  const T* const p = z + row * ld;
  const int head = head_of(p, k), nv = (k - head) / N, tail = head + nv * N;
  float m = -INFINITY, s = 0.f;
  auto take = [&](const auto& vs) {
    constexpr int V = sizeof(vs) / sizeof(vs[0]);
    float x[V * N], top = m;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int t = 0; t < N; ++t) x[i * N + t] = to_f(vs[i].x[t]), top = fmaxf(top, x[i * N + t]);
    const float ref = top == -INFINITY ? 0.f : top;
    s *= __builtin_amdgcn_exp2f((m - ref) * kLog2e);
#pragma unroll
    for (int i = 0; i < V * N; ++i) s += __builtin_amdgcn_exp2f((x[i] - ref) * kLog2e);
    m = top;
  };
  for (int e = tid; e < head; e += 256) join(m, s, to_f(p[e]), 1.f);
  for (int e = tail + tid; e < k; e += 256) join(m, s, to_f(p[e]), 1.f);
  // eight 16-byte loads of a thread in flight, rescaled once for all eight
  const T* const q = p + head;
  int v = tid;
  for (; v + 7 * 256 < nv; v += 8 * 256) {
    Vec<T> a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = load_vec(q + (int64_t)(v + 256 * i) * N);
    take(a);
  }
  for (; v < nv; v += 256) {
    const Vec<T> a[1] = {load_vec(q + (int64_t)v * N)};
    take(a);
  }
  const float top = wave_max(m);
  const float ref = top == -INFINITY ? 0.f : top;
  s = wave_sum(s * __builtin_amdgcn_exp2f((m - ref) * kLog2e));
  if ((tid & 63) == 0) sm[tid >> 6] = top, ss[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    m = sm[0], s = ss[0];
    for (int w = 1; w < 4; ++w) join(m, s, sm[w], ss[w]);
    const int a = act[row];
    const bool counts = a >= 0 && a < k;
    finish_row(m, s, counts ? to_f(p[a]) : 0.f, counts, row_lse + row, picked + i);
  }
}

__device__ __forceinline__ double wave_sum_f64(double x) {
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

template <class L>
__device__ __forceinline__ double margin_of(const L* logp2, const float* ref, int pair, float beta) {
  const double rw = ref ? (double)ref[2 * pair] : 0.0, rl = ref ? (double)ref[2 * pair + 1] : 0.0;
  return (double)beta * (((double)logp2[0] - rw) - ((double)logp2[1] - rl));
}

// A block of two waves per pair, a wave per answer.
__global__ __launch_bounds__(128) void pref_pairs_kernel(const double* __restrict__ picked,
                                                        const int32_t* __restrict__ offs, const float* ref, float beta,
                                                        float eps, float* __restrict__ logp, float* __restrict__ loss) {
  __shared__ double both[2];
  const int pair = blockIdx.x, w = threadIdx.x >> 6, lane = threadIdx.x & 63, ans = 2 * pair + w;
  double x = 0.0;
  for (int r = offs[ans] + lane; r < offs[ans + 1]; r += 64) x += picked[r];
  x = wave_sum_f64(x);
  if (lane == 0) both[w] = x, logp[ans] = (float)x;
  __syncthreads();
  if (threadIdx.x == 0) {
    const double m = margin_of(both, ref, pair, beta);
    const double tail = log1p(exp(-fabs(m)));
    // (a weight of 0 drops its term: an action of probability 0 makes m infinite)
    const double sure = (1.0 - (double)eps) * (fmax(-m, 0.0) + tail), other = (double)eps * (fmax(m, 0.0) + tail);
    loss[pair] = (float)(eps == 0.f ? sure : eps == 1.f ? other : sure + other);
  }
}

__global__ __launch_bounds__(128) void pref_coef_kernel(const int32_t* __restrict__ offs, const float* ref,
                                                       const float* __restrict__ logp, const float* dloss, float beta,
                                                       float eps, float* __restrict__ coef) {
  const int pair = blockIdx.x, w = threadIdx.x >> 6, lane = threadIdx.x & 63, ans = 2 * pair + w;
  const double m = margin_of(logp + 2 * pair, ref, pair, beta);
  const double slope = eps * (1.0 / (1.0 + exp(-m))) - (1.0 - (double)eps) * (1.0 / (1.0 + exp(m)));
  const float c = (float)((w ? -slope : slope) * (double)beta * (double)dloss[pair]);
  for (int r = offs[ans] + lane; r < offs[ans + 1]; r += 64) coef[r] = c;
}

template <class T>
__global__ __launch_bounds__(256) void pref_grad_narrow(const T* __restrict__ z, int64_t ld, int k, int W,
                                                       const int32_t* __restrict__ act, int64_t row0, int64_t n,
                                                       const float* __restrict__ row_lse,
                                                       const float* __restrict__ coef, T* __restrict__ dz,
                                                       int64_t ldd) {
  const int j = threadIdx.x & (W - 1);
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / W;
  if (i >= n || j >= k) return;
  const int a = act[row0 + i];
  const float l = row_lse[row0 + i];
  float g = 0.f;
  if (a >= 0 && a < k && l != -INFINITY) g = coef[i] * ((j == a ? 1.f : 0.f) - expf(to_f(z[(row0 + i) * ld + j]) - l));
  dz[(row0 + i) * ldd + j] = (T)g;
}

template <class T>
__global__ __launch_bounds__(256) void pref_grad_scalar(const T* __restrict__ z, int64_t ld,
                                                       const int32_t* __restrict__ act, int64_t row0, int64_t n,
                                                       const float* __restrict__ coef, T* __restrict__ dz,
                                                       int64_t ldd) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int a = act[row0 + i];
  const float s = to_f(z[(row0 + i) * ld]);
  // 1 - sigmoid(s) = sigmoid(-s): no difference of near equals
  float g = 0.f;
  if (a == 1) g = coef[i] * (1.f / (1.f + expf(s)));
  else if (a == 0) g = -coef[i] * (1.f / (1.f + expf(-s)));
  dz[(row0 + i) * ldd] = (T)g;
}

template <class T>
__global__ __launch_bounds__(256) void pref_grad_wide(const T* __restrict__ z, int64_t ld, int k,
                                                     const int32_t* __restrict__ act, int64_t row0,
                                                     const float* __restrict__ row_lse, const float* __restrict__ coef,
                                                     T* __restrict__ dz, int64_t ldd) {
  constexpr int N = Vec<T>::N;
  const int tid = threadIdx.x;
  // last row first: what the forward read last may still be in the caches
  const int64_t i = (int64_t)gridDim.x - 1 - blockIdx.x, row = row0 + i;
  const T* const p = z + row * ld;
  T* const o = dz + row * ldd;
  const int a = act[row];
  const float l = row_lse[row];
  const bool counts = a >= 0 && a < k && l != -INFINITY;
  const float c = counts ? coef[i] : 0.f, ref = counts ? l : 0.f;
  auto grad = [&](float x, int e) {
    const float soft = __builtin_amdgcn_exp2f((x - ref) * kLog2e);
    return counts ? c * ((e == a ? 1.f : 0.f) - soft) : 0.f;
  };
  // 16-byte pieces where logits and gradients are aligned alike
  const bool alike = (((uintptr_t)p ^ (uintptr_t)o) & 15) == 0;
  const int head = alike ? head_of(p, k) : k, nv = (k - head) / N, tail = head + nv * N;
  for (int e = tid; e < head; e += 256) o[e] = (T)grad(to_f(p[e]), e);
  for (int e = tail + tid; e < k; e += 256) o[e] = (T)grad(to_f(p[e]), e);
#pragma unroll 4
  for (int v = tid; v < nv; v += 256) {
    const int e = head + v * N;
    const Vec<T> x = load_vec(p + e);
    Vec<T> y;
#pragma unroll
    for (int t = 0; t < N; ++t) y.x[t] = (T)grad(to_f(x.x[t]), e + t);
    *reinterpret_cast<u32x4_t*>(o + e) = __builtin_bit_cast(u32x4_t, y);
  }
}

int lanes_for(int k) {
  int w = 2;
  while (w < k) w <<= 1;
  return w;
}

// Rows of a launch: a grid holds fewer than 2^32 threads, 256 of a wide row.
constexpr int64_t kRowsPerLaunch = 1 << 23;

template <class T>
hipError_t rows(const T* z, int64_t ld, int k, const int32_t* act, int64_t row0, int64_t n, float* lse, double* picked,
                hipStream_t s) {
  if (k == 1) {
    pref_rows_scalar<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(z, ld, act, row0, n, lse, picked);
  } else if (k <= 64) {
    const int W = lanes_for(k), per = 256 / W;
    pref_rows_narrow<T><<<(unsigned)((n + per - 1) / per), 256, 0, s>>>(z, ld, k, W, act, row0, n, lse, picked);
  } else {
    pref_rows_wide<T><<<(unsigned)n, 256, 0, s>>>(z, ld, k, act, row0, lse, picked);
  }
  return hipGetLastError();
}

template <class T>
hipError_t grad(const T* z, int64_t ld, int k, const int32_t* act, int64_t row0, int64_t n, const float* lse,
                const float* coef, T* dz, int64_t ldd, hipStream_t s) {
  if (k == 1) {
    pref_grad_scalar<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(z, ld, act, row0, n, coef, dz, ldd);
  } else if (k <= 64) {
    const int W = lanes_for(k), per = 256 / W;
    pref_grad_narrow<T><<<(unsigned)((n + per - 1) / per), 256, 0, s>>>(z, ld, k, W, act, row0, n, lse, coef, dz, ldd);
  } else {
    pref_grad_wide<T><<<(unsigned)n, 256, 0, s>>>(z, ld, k, act, row0, lse, coef, dz, ldd);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pref_offsets(int32_t* dst, const PrefOffsets& a, hipStream_t s) {
  pref_offsets_kernel<<<1, 256, 0, s>>>(dst, a);
  return hipGetLastError();
}
hipError_t launch_pref_rows(bool bf, const void* logits, int64_t ld, int32_t k, const int32_t* act, int64_t row0,
                            int64_t n, float* row_lse, double* picked, hipStream_t s) {
  hipError_t e = hipSuccess;
  for (int64_t r = 0; r < n && e == hipSuccess; r += kRowsPerLaunch) {
    const int64_t m = n - r < kRowsPerLaunch ? n - r : kRowsPerLaunch;
    e = bf ? rows((const bf16*)logits, ld, k, act, row0 + r, m, row_lse, picked + r, s)
           : rows((const float*)logits, ld, k, act, row0 + r, m, row_lse, picked + r, s);
  }
  return e;
}
hipError_t launch_pref_pairs(const double* picked, const int32_t* offs, int32_t n_pairs, const float* ref, float beta,
                             float eps, float* logp, float* loss, hipStream_t s) {
  pref_pairs_kernel<<<n_pairs, 128, 0, s>>>(picked, offs, ref, beta, eps, logp, loss);
  return hipGetLastError();
}
hipError_t launch_pref_coef(const int32_t* offs, int32_t n_pairs, const float* ref, const float* logp,
                            const float* dloss, float beta, float eps, float* coef, hipStream_t s) {
  pref_coef_kernel<<<n_pairs, 128, 0, s>>>(offs, ref, logp, dloss, beta, eps, coef);
  return hipGetLastError();
}
hipError_t launch_pref_grad(bool bf, const void* logits, int64_t ld, int32_t k, const int32_t* act, int64_t row0,
                            int64_t n, const float* row_lse, const float* coef, void* dlogits, int64_t ldd,
                            hipStream_t s) {
  hipError_t e = hipSuccess;
  for (int64_t r = 0; r < n && e == hipSuccess; r += kRowsPerLaunch) {
    const int64_t m = n - r < kRowsPerLaunch ? n - r : kRowsPerLaunch;
    e = bf ? grad((const bf16*)logits, ld, k, act, row0 + r, m, row_lse, coef + r, (bf16*)dlogits, ldd, s)
           : grad((const float*)logits, ld, k, act, row0 + r, m, row_lse, coef + r, (float*)dlogits, ldd, s);
  }
  return e;
}

}  // namespace tx
