// Per-stage HIP-event timing shared by the sources that hold entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <mutex>
#include <vector>

#include "host.hpp"

namespace tri {

struct Profiler {
  std::mutex mu;
  bool on = false;
  struct Rec { int stage; hipEvent_t a, b; };
  std::vector<Rec> pending;
  std::vector<hipEvent_t> pool;
  int launches[ST_COUNT] = {};
  double ms[ST_COUNT] = {};
  hipEvent_t get() {
    if (!pool.empty()) { hipEvent_t e = pool.back(); pool.pop_back(); return e; }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
  }
};
inline Profiler& prof() { static Profiler p; return p; }

// Records an event pair around one stage when profiling is on.
struct StageTimer {
  int stage;
  hipStream_t s;
  hipEvent_t a = nullptr, b = nullptr;
  StageTimer(int st, hipStream_t str, bool timed = true) : stage(st), s(str) {
    Profiler& p = prof();
    if (!timed || !p.on) return;
    std::lock_guard<std::mutex> g(p.mu);
    a = p.get();
    b = p.get();
    if (a && b) hipEventRecord(a, s);
  }
  ~StageTimer() {
    if (!a || !b) return;
    Profiler& p = prof();
    hipEventRecord(b, s);
    std::lock_guard<std::mutex> g(p.mu);
    p.pending.push_back({stage, a, b});
  }
};

#define TRI_HIP(expr)                              \
  do {                                             \
    if ((expr) != hipSuccess) return TRI_ERR_HIP;  \
  } while (0)

}  // namespace tri
