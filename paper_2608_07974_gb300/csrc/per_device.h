// What is found out once for every device that a process uses (host side, no CUDA in it).
#pragma once
#include <atomic>
#include <mutex>

namespace zl {

template <typename T, int kDevices = 64>
class PerDevice {
 public:
  // The value of device dev. make(T&) finds it out when the device is first asked for, while other threads wait, and again the
  // next time if it returns false. NULL without a value.
  template <typename F>
  const T* get(int dev, F&& make) {
    if (dev < 0 || dev >= kDevices) return nullptr;
    if (!ready_[dev].load(std::memory_order_acquire)) {
      std::lock_guard<std::mutex> lock(mutex_);
      if (!ready_[dev].load(std::memory_order_relaxed)) {
        if (!make(value_[dev])) return nullptr;
        ready_[dev].store(true, std::memory_order_release);
      }
    }
    return &value_[dev];
  }

 private:
  std::mutex mutex_;
  std::atomic<bool> ready_[kDevices] = {};
  T value_[kDevices] = {};
};

}  // namespace zl
