// Something that is done once on every device a process uses (a kernel's attributes belong to a device).  Plain C++, so that it
// is tested without a GPU.
#pragma once

#include <atomic>
#include <cstdint>

namespace zq {

class DeviceOnce {
  std::atomic<uint64_t> done_{0};

 public:
  // `f` on a device's first call, and again until it has returned true there; whether it has.  (Threads that arrive together may
  // each run it, so it must not mind being repeated.)
  template <typename F>
  bool run(int device, F&& f) {
    if (device < 0 || device >= 64) return f();
    const uint64_t bit = uint64_t(1) << device;
    if (done_.load(std::memory_order_acquire) & bit) return true;
    if (!f()) return false;
    done_.fetch_or(bit, std::memory_order_release);
    return true;
  }
};

}  // namespace zq
