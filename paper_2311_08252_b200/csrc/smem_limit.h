// What each kernel's dynamic shared-memory limit was raised to, per device.  Host code without CUDA.
#pragma once
#include <stddef.h>

#include <atomic>
#include <mutex>

namespace rest {

template <int kDevices, int kSlots>
class SmemLimits {
 public:
  // Makes the limit at least `bytes` by raise(), which returns 0 or an error.  Threads whose calls need different
  // sizes come here at the same time: one at a time raises, and only upwards, so that no limit ends up
  // below what is remembered of it.
  template <typename Raise>
  int ensure(int device, int slot, size_t bytes, Raise raise) {
    if (device < 0 || device >= kDevices || slot < 0 || slot >= kSlots) return raise();
    std::atomic<size_t>& have = set_[device][slot];
    if (have.load(std::memory_order_acquire) >= bytes) return 0;
    std::lock_guard<std::mutex> lock(mutex_);
    if (have.load(std::memory_order_relaxed) >= bytes) return 0;
    const int error = raise();
    if (error == 0) have.store(bytes, std::memory_order_release);
    return error;
  }

 private:
  std::mutex mutex_;
  std::atomic<size_t> set_[kDevices][kSlots] = {};
};

}  // namespace rest
