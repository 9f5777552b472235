// What the files of the C ABI share: status and message of a failed call,
// argument checks, and the per-kernel event timing.  Host only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <mutex>
#include <string>
#include <vector>

#include "dtst.h"

namespace dtst {

// Message of the last failed call on this thread ("" after a good one).
std::string& last_error();

dtst_status fail(dtst_status s, const std::string& msg);
dtst_status ok();
dtst_status device_status(int e, const char* what);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
dtst_status check_ptr(const void* ptr, const char* name);

#define DTST_TRY(expr)                 \
  do {                                 \
    dtst_status s_ = (expr);           \
    if (s_ != DTST_OK) return s_;      \
  } while (0)

// ---- per-kernel event timing (dtst_profile_enable / dtst_profile_collect) ----
enum KernelRole { K_FWD_TZ, K_AXIS_FWD_Y, K_AXIS_FWD_X, K_AXIS_INV_X, K_AXIS_INV_Y, K_INV_ZT, K_MIX, K_MIX_H,
                  K_WGRAD, K_BLOCK, K_FWD_TZY, K_INV_YZT, K_POINTWISE, K_INV_ZT_BLOCK, K_NORM, K_NORM_ADJ,
                  K_QUANTISE, K_PRODUCT, K_RECUR, K_RECUR_ADJ, K_COUNT };
extern const char* const kRoleNames[K_COUNT];

struct Profiler {
  std::mutex mu;
  bool on = false;
  struct Rec {
    int role;
    hipEvent_t a, b;
  };
  std::vector<Rec> pending;
  std::vector<hipEvent_t> pool;
  double total_ms[K_COUNT] = {};
  int64_t launches[K_COUNT] = {};
  hipEvent_t get() {
    if (!pool.empty()) {
      hipEvent_t e = pool.back();
      pool.pop_back();
      return e;
    }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
  }
};
Profiler& prof();

// Runs one launcher; when profiling is on, brackets it with events on `stream`.
template <class F>
int timed(int role, void* stream, F&& launch) {
  Profiler& P = prof();
  bool on;
  {
    std::lock_guard<std::mutex> lk(P.mu);
    on = P.on;
  }
  if (!on) return launch();
  hipEvent_t a, b;
  {
    std::lock_guard<std::mutex> lk(P.mu);
    a = P.get();
    b = P.get();
  }
  if (a == nullptr || b == nullptr) return launch();
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipEventRecord(a, s);
  const int e = launch();
  (void)hipEventRecord(b, s);
  std::lock_guard<std::mutex> lk(P.mu);
  P.pending.push_back({role, a, b});
  return e;
}

}  // namespace dtst
