// What mpt_kv_check has told of the events that kernels count on a device.
// Plain C++, so that it is tested without a GPU.
#pragma once

#include <atomic>
#include <cstdint>

namespace mpt {

// The kernels add to a count that nothing clears, and a call that reads it
// compares it with what was told before: an event between one call's read and
// its answer, on whatever stream, is news to the next call, and of two calls
// that read the same event at least one tells of it.
class Reported {
 public:
  // Whether `count`, as read on `device`, has events that no call told of; this one does then.
  bool news(int device, uint32_t count) {
    if (device < 0 || device >= kDevices) return count != 0;
    uint32_t told = told_[device].load();
    while ((int32_t)(count - told) > 0)
      if (told_[device].compare_exchange_weak(told, count)) return true;
    return false;
  }

 private:
  static constexpr int kDevices = 64;
  std::atomic<uint32_t> told_[kDevices] = {};
};

}  // namespace mpt
