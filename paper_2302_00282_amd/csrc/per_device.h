// What is done once for each GPU of a process.  (Behind the runtime's header, or one that declares what is used of it here.)
#pragma once
#include <atomic>
#include <stdint.h>

namespace xenos {

// The devices for which it has been done.  (Done twice is no harm: two threads' first calls may both find it undone, and so does every call on a device beyond the 64th.)
class PerDevice {
  std::atomic<uint64_t> done_{0};

 public:
  bool done(int device) const { return device >= 0 && device < 64 && (done_.load(std::memory_order_acquire) >> device & 1); }
  void set(int device) {
    if (device >= 0 && device < 64) done_.fetch_or(uint64_t{1} << device, std::memory_order_release);
  }
};

// A kernel's limit of dynamic LDS is raised once on each device, which has the function's attributes for itself: to all of a unit's memory where its launches differ in
// their need.  (Raised to what the launch at hand needs, two threads' first launches could leave the smaller limit behind.)
constexpr int kLdsPerUnit = 160 * 1024;
template <typename F>
inline hipError_t raise_lds_limit(F* kernel, PerDevice& raised, int bytes = kLdsPerUnit) {
  int device = -1;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess || raised.done(device)) return e;
  e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) raised.set(device);
  return e;
}

}  // namespace xenos
