// What has to be done once on every device: a kernel's attributes belong to the function on the device that is current, and a process
// may use several.
#pragma once
#include <atomic>
#include <cstdint>

namespace kvr {

class OncePerDevice {
 public:
  // Runs action() (0: done) unless it was done on this device before.  A failure is returned and not kept: the next call tries
  // again.  Threads may come together: the action is run by each that finds it undone.  Devices from 64 on: run every time.
  template <class Action>
  auto operator()(int device, Action action) -> decltype(action()) {
    using Status = decltype(action());
    const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;
    if (done_.load(std::memory_order_acquire) & bit) return Status(0);
    const Status status = action();
    if (status == Status(0)) done_.fetch_or(bit, std::memory_order_release);
    return status;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

}  // namespace kvr
