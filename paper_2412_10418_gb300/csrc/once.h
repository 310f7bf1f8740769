// once.h -- a step that is done once on each device, such as a kernel's attributes, which belong to a device.
#pragma once

#include <atomic>
#include <cstdint>

namespace cdsl {

// step() returns 0 where it has succeeded; a failure is returned and not kept. Threads may both take the step at first.
class OncePerDevice {
 public:
  template <typename F>
  auto operator()(int device, F&& step) -> decltype(step()) {
    const uint64_t bit = (unsigned)device < 64u ? 1ull << device : 0ull;   // (beyond them: every time)
    if (done_.load(std::memory_order_acquire) & bit) return {};
    const auto result = step();
    if (result == decltype(step()){}) done_.fetch_or(bit, std::memory_order_release);
    return result;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

}  // namespace cdsl
