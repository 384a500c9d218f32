// What a kernel has been allowed of dynamic LDS, by device.
#pragma once

#include <stddef.h>

#include <atomic>
#include <mutex>

namespace bacon {

// The largest grant of one kernel on each device.  A grant belongs to a device's
// copy of the kernel: one device's says nothing about another's.
class LdsGrants {
 public:
  static constexpr size_t kFree = 64 * 1024;   // bytes that need no grant

  // Has allow(bytes) called where the device has not granted as much yet, and
  // returns its status: 0, or an error, after which the next call asks again.
  template <class Allow>
  int grant(int device, size_t bytes, Allow allow) {
    if (bytes <= kFree) return 0;
    std::atomic<size_t> *held = device >= 0 && device < kDevices ? &held_[device] : nullptr;
    if (held && bytes <= *held) return 0;
    std::lock_guard<std::mutex> lock(mutex_);  // a grant replaces the last: the largest has to be the last
    if (held && bytes <= *held) return 0;
    const int status = allow(bytes);
    if (status == 0 && held) *held = bytes;
    return status;
  }

 private:
  static constexpr int kDevices = 64;          // devices past these are asked every time
  std::atomic<size_t> held_[kDevices] = {};
  std::mutex mutex_;
};

}  // namespace bacon
