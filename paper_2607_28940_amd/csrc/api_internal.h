// What the C entry points of api.cpp and train.cpp share: the error message of
// the calling thread and the per-kernel timing of a launch.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

namespace tx {

// Sets the calling thread's message (tx_last_error) and returns code.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

enum KClass {
  K_GEMM_QKV, K_GEMM_O, K_GEMM_XQ, K_GEMM_XO, K_GEMM_FFN1, K_GEMM_FFN2, K_SELF_ATTN, K_CROSS_ATTN, K_LAYERNORM,
  K_LN_SCORE, K_COPY, K_ENC_GEMM, K_ENC_ATTN, K_ENC_LAYERNORM, K_SCATTER, K_XKV_GEMM, K_POOL,
  K_TRAIN_FWD, K_TRAIN_DQ, K_TRAIN_DKV, K_TRAIN_PREF, K_COUNT
};

// An event pair around a launch on its stream while tx_profile_enable is on.
struct ProfScope {
  int cls;
  hipStream_t st;
  double fl, by;
  hipEvent_t a = nullptr;
  ProfScope(int c, hipStream_t s, double f, double b);
  ~ProfScope();
};

inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

// Lays sub-buffers out in one device region (256-byte aligned); with a null
// base it only measures.
struct Carver {
  char* base;
  size_t off = 0;
  explicit Carver(void* b) : base((char*)b) {}
  template <class P>
  P take(size_t bytes) {
    const size_t o = align_up(off);
    off = o + bytes;
    return base ? (P)(base + o) : (P) nullptr;
  }
};

}  // namespace tx

#define TX_HIP(expr)                                                                        \
  do {                                                                                      \
    hipError_t e_ = (expr);                                                                 \
    if (e_ != hipSuccess) return fail(TX_E_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

#define TX_CHECK(code)           \
  do {                           \
    int c_ = (code);             \
    if (c_ != TX_OK) return c_;  \
  } while (0)

#define TX_LAUNCH(cls, fl, by, expr) \
  do {                               \
    ProfScope ps_((cls), st, (fl), (by)); \
    TX_HIP(expr);                    \
  } while (0)
