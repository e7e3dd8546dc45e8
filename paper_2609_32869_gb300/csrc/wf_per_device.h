// What a process sets up once for each device that it uses: a kernel's
// attributes, or a property read once.  Plain C++, so that the host tests
// include it.
#pragma once
#include <atomic>
#include <mutex>

namespace wf {

class PerDevice {
 public:
  // The device's value: set_up()'s for the first call that succeeds on it.
  // set_up runs with that device current and returns 0 where it fails, which
  // is not kept.
  template <typename F>
  int get(int device, F set_up) {
    if (device < 0 || device >= kMax) return set_up();
    if (const int v = value_[device].load(std::memory_order_acquire)) return v;
    std::lock_guard<std::mutex> lock(mu_);
    if (const int v = value_[device].load(std::memory_order_relaxed)) return v;
    const int v = set_up();
    value_[device].store(v, std::memory_order_release);
    return v;
  }

 private:
  static constexpr int kMax = 64;
  std::mutex mu_;
  std::atomic<int> value_[kMax] = {};
};

}  // namespace wf
