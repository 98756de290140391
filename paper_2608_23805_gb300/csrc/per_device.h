// Numbers that are asked for once on each device (a kernel's residency, say): host
// code that runs on whichever device is current keeps them by its number.
#pragma once

#include <atomic>

namespace msi {

template <int KEYS>
class PerDevice {
 public:
  static constexpr int kDevices = 64;
  // *value of `key` on device dev; ask(value) tells it and returns 0 where it can.  A
  // device past kDevices is asked about each time.
  template <class Ask>
  auto get(int dev, int key, int* value, Ask ask) -> decltype(ask(value)) {
    const bool keep = dev >= 0 && dev < kDevices;
    if (keep) {
      *value = kept_[dev][key].load(std::memory_order_relaxed) - 1;
      if (*value >= 0) return decltype(ask(value))();
    }
    const auto e = ask(value);
    if (keep && !e && *value >= 0) kept_[dev][key].store(*value + 1, std::memory_order_relaxed);
    return e;
  }

 private:
  std::atomic<int> kept_[kDevices][KEYS] = {};  // the value and 1; 0: not asked yet
};

}  // namespace msi
