// What has to be done once on every device before its first use there.
#pragma once

#include <stdint.h>

#include <atomic>

namespace hyenand {

// f() once for each device, again where it failed; 0 is success.  Threads that come
// at the same time may each run it, so f must do no harm a second time.
class DeviceOnce {
 public:
  template <typename F>
  auto operator()(int device, F f) -> decltype(f()) {
    const uint64_t bit = device >= 0 && device < 64 ? uint64_t(1) << device : 0;  // 0: each time
    if (done_.load(std::memory_order_acquire) & bit) return decltype(f())(0);
    const auto e = f();
    if (e == 0) done_.fetch_or(bit, std::memory_order_release);
    return e;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

}  // namespace hyenand
