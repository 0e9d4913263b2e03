// Set-up that a device needs once (kernel attributes apply to the device that is current).
#pragma once
#include <atomic>

namespace spd {

class DeviceOnce {
 public:
  // Calls set() unless it has returned 0 for this device before, and returns its result. Threads may call at the same
  // time, and then may all call set(): it must not mind. No lock, and nothing that throws.
  template <typename F>
  int run(int device, F&& set) {
    const unsigned long long bit = device >= 0 && device < 64 ? 1ull << device : 0;
    if (done_.load(std::memory_order_acquire) & bit) return 0;
    const int rc = set();
    if (rc == 0) done_.fetch_or(bit, std::memory_order_release);
    return rc;
  }

 private:
  std::atomic<unsigned long long> done_{0};
};

}  // namespace spd
