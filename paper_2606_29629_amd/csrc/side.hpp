// A second stream per device, on which one kernel of a call runs beside another.
#pragma once
#include <hip/hip_runtime.h>

#include <mutex>

namespace tri {

// A second stream per device, on which a mixed batch's split-KV attention
// (the single-token sequences) runs beside the flash attention of its
// multi-token sequences: both read the projected q and the cache, and they
// write disjoint output rows and disjoint partials.  Created on first use
// (default priority, non-blocking); the fork and join events are recorded and
// waited on under the device's lock, so concurrent callers cannot pair one
// caller's record with another's wait.
struct SideStream {
  std::mutex mu;
  hipStream_t s = nullptr;
  hipEvent_t fork = nullptr, join = nullptr;
  bool failed = false;  // creation failed once (e.g. under graph capture): run serially
};
constexpr int kMaxSideDevices = 64;
// The side stream of the current device, or nullptr (run on the caller's
// stream) when the caller's stream belongs to another device.
inline SideStream* side_stream(hipStream_t caller) {
  static SideStream ss[kMaxSideDevices];
  int dev = -1, sdev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxSideDevices) return nullptr;
  if (caller && (hipStreamGetDevice(caller, &sdev) != hipSuccess || sdev != dev)) {
    (void)hipGetLastError();
    return nullptr;
  }
  return &ss[dev];
}
// With the device's lock held: makes sure the stream and events exist; false
// means "run on the caller's stream".  No stream is created while the
// caller's stream is being captured into a graph (creating one could
// invalidate the capture); an existing side stream joins the capture through
// the fork and join events.
inline bool side_ready(SideStream& x, hipStream_t caller) {
  if (x.s) return true;
  if (x.failed) return false;
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(caller, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) {
    (void)hipGetLastError();
    return false;
  }
  hipStream_t st = nullptr;
  hipEvent_t f = nullptr, j = nullptr;
  if (hipStreamCreateWithFlags(&st, hipStreamNonBlocking) == hipSuccess &&
      hipEventCreateWithFlags(&f, hipEventDisableTiming) == hipSuccess &&
      hipEventCreateWithFlags(&j, hipEventDisableTiming) == hipSuccess) {
    x.s = st;
    x.fork = f;
    x.join = j;
    return true;
  }
  if (f) (void)hipEventDestroy(f);
  if (st) (void)hipStreamDestroy(st);
  (void)hipGetLastError();  // clear the failed call's error
  x.failed = true;
  return false;
}

// Whether the side stream may join the caller's work: not while it belongs to a capture
// that is still open and is not the caller's (of another stream, by another thread).
inline bool side_free(const SideStream& x, hipStream_t caller) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone, ss = cs;
  unsigned long long ci = 0, si = 0;
  if (hipStreamGetCaptureInfo(x.s, &ss, &si) != hipSuccess ||
      hipStreamGetCaptureInfo(caller, &cs, &ci) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return ss == hipStreamCaptureStatusNone || (cs == ss && ci == si);
}

// One fork of the caller's stream: begin() makes `stream` the side stream, at the caller's
// point, or the caller's own where there is none; end() makes the caller wait for it.  The
// device's lock is held in between.
struct Fork {
  hipStream_t caller = nullptr, stream = nullptr;
  SideStream* side = nullptr;
  std::unique_lock<std::mutex> lock;
  hipError_t begin(hipStream_t s) {
    caller = stream = s;
    SideStream* x = side_stream(s);
    if (!x) return hipSuccess;
    lock = std::unique_lock<std::mutex>(x->mu);
    if (!side_ready(*x, s) || !side_free(*x, s)) return hipSuccess;
    hipError_t e = hipEventRecord(x->fork, s);
    if (e == hipSuccess) e = hipStreamWaitEvent(x->s, x->fork, 0);
    if (e != hipSuccess) return e;
    side = x;
    stream = x->s;
    return hipSuccess;
  }
  hipError_t end() {
    hipError_t e = hipSuccess;
    if (side) {
      e = hipEventRecord(side->join, side->s);
      if (e == hipSuccess) e = hipStreamWaitEvent(caller, side->join, 0);
      side = nullptr;
    }
    if (lock.owns_lock()) lock.unlock();
    return e;
  }
};

}  // namespace tri
