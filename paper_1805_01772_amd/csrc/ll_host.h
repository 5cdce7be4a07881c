// Host-side helpers shared by the entry points (errors, device selection).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lstmloop.h"

namespace ll {

// Sets the calling thread's message (ll_last_error) and returns s.
ll_status fail(ll_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// hipMalloc with the library's errors; zero bytes allocate a little.
ll_status dalloc(void** out, size_t bytes, const char* what);

// LL_EINVAL unless `device` is one of the machine's.
ll_status check_device(int device);

// Waits for the device, then reads the error word at `word` into *out (may be
// NULL) and clears it.
ll_status read_error_word(int* word, int32_t* out);

// What a plan's creation wrote (on the default stream) is there for calls on any stream,
// also for those that do not wait for the default one.
inline ll_status wait_created() {
  const hipError_t e = hipStreamSynchronize(nullptr);
  return e == hipSuccess ? LL_OK : fail(LL_EHIP, "waiting for the plan's memory failed: %s", hipGetErrorString(e));
}

// Work-items of a launch are counted in 32 bits: work-groups of `threads` that one holds.
constexpr int64_t max_groups(int threads) { return (((int64_t)1 << 32) - 1) / threads; }

inline bool aligned_to(const void* p, unsigned bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool aligned16(const void* p) { return aligned_to(p, 16); }

class DeviceGuard {
 public:
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev_) != hipSuccess) prev_ = -1;
    if (prev_ != dev) (void)hipSetDevice(dev);
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev_ >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev_) (void)hipSetDevice(prev_);
  }

 private:
  int prev_ = -1;
};

}  // namespace ll

#define LL_HIP(call)                                                              \
  do {                                                                            \
    hipError_t e_ = (call);                                                       \
    if (e_ != hipSuccess)                                                         \
      return ll::fail(LL_EHIP, "%s failed: %s", #call, hipGetErrorString(e_));    \
  } while (0)

// Refuses an argument that is not aligned to `bytes`.
#define LL_ALIGNED(p, bytes)                                                      \
  do {                                                                            \
    if (!ll::aligned_to(p, bytes))                                                \
      return ll::fail(LL_EINVAL, "%s = %p is not %d-byte aligned", #p, (const void*)(p), (int)(bytes)); \
  } while (0)

#define LL_STATUS(call)         \
  do {                          \
    ll_status st_ = (call);     \
    if (st_ != LL_OK) return st_; \
  } while (0)
