// The few runtime calls of staging.h on two devices that exist in host memory only.  Copies are
// done when an event behind them is waited for, so that a buffer used again too early shows.
#pragma once
#include <cstdlib>
#include <cstring>
#include <functional>
#include <vector>

enum hipError_t { hipSuccess = 0, hipErrorInvalidHandle = 400 };
enum hipMemcpyKind { hipMemcpyHostToDevice = 1 };
constexpr unsigned hipHostMallocDefault = 0, hipEventDisableTiming = 2;

struct FakeStream {
  int device;
  std::vector<std::function<void()>> work;
};
struct FakeEvent {
  int device;
  FakeStream *at = nullptr;
};
using hipStream_t = FakeStream *;
using hipEvent_t = FakeEvent *;

inline int fake_device = 0, fake_waits = 0, fake_buffers = 0;

inline hipError_t hipGetDevice(int *d) {
  *d = fake_device;
  return hipSuccess;
}
inline hipError_t hipHostMalloc(void **p, size_t n, unsigned) {
  *p = std::malloc(n);
  ++fake_buffers;
  return hipSuccess;
}
inline hipError_t hipHostFree(void *p) {
  std::free(p);
  --fake_buffers;
  return hipSuccess;
}
inline hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) {
  *e = new FakeEvent{fake_device};
  return hipSuccess;
}
inline hipError_t hipMemcpyAsync(void *dst, const void *src, size_t n, hipMemcpyKind, hipStream_t s) {
  if (s->device != fake_device) return hipErrorInvalidHandle;
  s->work.push_back([=] { std::memcpy(dst, src, n); });
  return hipSuccess;
}
inline hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
  if (e->device != s->device) return hipErrorInvalidHandle;   // as the runtime has it
  e->at = s;
  return hipSuccess;
}
inline void fake_finish(hipStream_t s) {
  for (auto &w : s->work) w();
  s->work.clear();
}
inline hipError_t hipEventSynchronize(hipEvent_t e) {
  ++fake_waits;
  if (e->at) fake_finish(e->at);
  return hipSuccess;
}
