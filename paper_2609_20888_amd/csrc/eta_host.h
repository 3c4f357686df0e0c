// Host helpers shared by the sources that hold entry points (eta_api.cpp,
// eta_train_api.cpp): the per-thread error string, small argument checks and the
// optional kernel timer.  Everything is inline, so each source can also be
// built without the other.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <mutex>
#include <string>
#include <vector>

#include "eta.h"
#include "eta_internal.h"

namespace eta {

inline thread_local std::string g_err;

inline eta_status_t fail(eta_status_t code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

inline eta_status_t ok() {
  g_err.clear();
  return ETA_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int elem_bytes(int dt) { return dt == ETA_DT_F32 ? 4 : 2; }

inline bool valid_dtype(int dt) { return dt == ETA_DT_F32 || dt == ETA_DT_BF16; }

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// ------------------------------------------------------------- kernel timer

struct Profiler {
  std::mutex mu;
  bool on = false;
  std::vector<hipEvent_t> pool;       // pairs: [2i] start, [2i+1] end
  std::vector<int> kinds;
  size_t used = 0;
  static constexpr size_t kMaxPairs = 65536;
};
inline Profiler& prof() {
  static Profiler p;
  return p;
}

inline void hook_fn(int kind, hipStream_t st, bool after) {
  Profiler& P = prof();
  std::lock_guard<std::mutex> lk(P.mu);
  if (!P.on) return;
  if (!after) {
    if (P.used >= Profiler::kMaxPairs) return;
    if (2 * P.used + 2 > P.pool.size()) {
      hipEvent_t a, b;
      if (hipEventCreate(&a) != hipSuccess) return;
      if (hipEventCreate(&b) != hipSuccess) { (void)hipEventDestroy(a); return; }
      P.pool.push_back(a);
      P.pool.push_back(b);
    }
    (void)hipEventRecord(P.pool[2 * P.used], st);
    P.kinds.push_back(kind);
  } else {
    if (P.kinds.size() != P.used + 1) return;
    (void)hipEventRecord(P.pool[2 * P.used + 1], st);
    ++P.used;
  }
}

inline LaunchHook active_hook() {
  Profiler& P = prof();
  std::lock_guard<std::mutex> lk(P.mu);
  return P.on ? hook_fn : nullptr;
}

}  // namespace eta
