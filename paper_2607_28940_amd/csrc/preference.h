// Launch functions of the preference loss (preference.hip).
#pragma once

#include "tx_internal.h"

namespace tx {

// Row offsets base, base + len[0], base + len[0] + len[1], .. (n lengths, n + 1
// offsets) as kernel arguments.
struct PrefOffsets {
  static constexpr int kLengths = 1536;
  int32_t base, n;
  uint16_t len[kLengths];
};
hipError_t launch_pref_offsets(int32_t* dst, const PrefOffsets& a, hipStream_t s);

// Per row r of row0 .. row0 + n - 1 with logits z [k] (k = 1: the scalar logit
// s, read as [0, s]): row_lse[r] = log sum exp z and picked[r - row0] = z[act] -
// lse, 0 for rows whose action lies outside the vocabulary or whose logits are
// all minus infinity.
hipError_t launch_pref_rows(bool bf, const void* logits, int64_t ld, int32_t k, const int32_t* act, int64_t row0,
                            int64_t n, float* row_lse, double* picked, hipStream_t s);
// Sums per answer (offs: 2 * n_pairs + 1 row offsets from row0) and the pairs' losses.
hipError_t launch_pref_pairs(const double* picked, const int32_t* offs, int32_t n_pairs, const float* ref, float beta,
                             float eps, float* logp, float* loss, hipStream_t s);
// coef[row - row0]: what a row's one-hot minus softmax is multiplied by.
hipError_t launch_pref_coef(const int32_t* offs, int32_t n_pairs, const float* ref, const float* logp,
                            const float* dloss, float beta, float eps, float* coef, hipStream_t s);
hipError_t launch_pref_grad(bool bf, const void* logits, int64_t ld, int32_t k, const int32_t* act, int64_t row0,
                            int64_t n, const float* row_lse, const float* coef, void* dlogits, int64_t ldd,
                            hipStream_t s);

}  // namespace tx
