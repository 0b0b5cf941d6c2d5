// How much dynamic shared memory a kernel has been allowed on each device.
#pragma once
#include <atomic>
#include <mutex>

namespace thinfer {

// The allowance is set for a kernel on a device and stays; one of these per kernel remembers the largest that has been set,
// so that a launch usually pays one look.  Check, setting and note are one step under a lock, and a smaller size is never
// set after a larger one: a thread that wants less cannot take from another what it has just been given.
class SmemAllowance {
 public:
  static constexpr int kMaxDevices = 64;
  // allow(bytes) sets the allowance on the device and says whether that worked.
  template <typename Allow>
  bool ensure(int device, int bytes, Allow allow) noexcept {
    if (device < 0 || device >= kMaxDevices) return allow(bytes);
    if (bytes <= largest_[device].load(std::memory_order_acquire)) return true;
    try {
      std::lock_guard<std::mutex> one(lock_);
      if (bytes <= largest_[device].load(std::memory_order_relaxed)) return true;
      if (!allow(bytes)) return false;
      largest_[device].store(bytes, std::memory_order_release);
      return true;
    } catch (...) {  // the lock could not be had
      return false;
    }
  }

 private:
  std::atomic<int> largest_[kMaxDevices] = {};
  std::mutex lock_;
};

}  // namespace thinfer
