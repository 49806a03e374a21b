// Pinned staging of host data on its way to the device, a buffer and an event for each device of a
// thread: an event is recorded on streams of its own device only, and a copy of one device does
// not wait for another's.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <vector>

namespace wisp {

class Staging {
 public:
  // `bytes` of `host` to `dst` in the order of `s`, a stream of the current device; NULL, or what failed
  const char *upload(const void *host, size_t bytes, void *dst, hipStream_t s) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) return "hipGetDevice failed";
    if ((size_t)dev >= slots_.size()) slots_.resize(dev + 1);
    Slot &g = slots_[dev];
    if (g.pending) {   // the buffer is used again once the copy before has finished
      if (hipEventSynchronize(g.ev) != hipSuccess) return "staging event sync failed";
      g.pending = false;
    }
    if (g.cap < bytes) {
      if (g.buf) (void)hipHostFree(g.buf);
      g.buf = nullptr;
      g.cap = 0;
      const size_t cap = std::max<size_t>(bytes, 1 << 16);
      if (hipHostMalloc(&g.buf, cap, hipHostMallocDefault) != hipSuccess) return "pinned staging allocation failed";
      g.cap = cap;
    }
    if (!g.ev && hipEventCreateWithFlags(&g.ev, hipEventDisableTiming) != hipSuccess) return "event creation failed";
    std::memcpy(g.buf, host, bytes);
    if (hipMemcpyAsync(dst, g.buf, bytes, hipMemcpyHostToDevice, s) != hipSuccess) return "descriptor upload failed";
    if (hipEventRecord(g.ev, s) != hipSuccess) return "event record failed";
    g.pending = true;
    return nullptr;
  }

 private:
  struct Slot {
    void *buf = nullptr;
    size_t cap = 0;
    hipEvent_t ev = nullptr;
    bool pending = false;
  };
  std::vector<Slot> slots_;   // by device
};

}  // namespace wisp
