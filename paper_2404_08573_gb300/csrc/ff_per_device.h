// What is set up or found out once for each device: attributes of kernels,
// how many of their clusters a GPU holds.
#pragma once

#include <atomic>
#include <mutex>

namespace ff {

template <typename T>
class PerDevice {
 public:
  // The value for device `dev`.  make(&value) forms it and returns an error
  // code, zero for success; a success is kept, a failure is returned and
  // tried again by the next call.
  template <typename F>
  auto get(int dev, T* out, F make) -> decltype(make(out)) {
    using E = decltype(make(out));
    const bool keeps = dev >= 0 && dev < kMost;
    if (keeps && slots_[dev].ready.load(std::memory_order_acquire)) {
      *out = slots_[dev].value;
      return E{};
    }
    T value{};
    const E e = make(&value);
    if (e != E{}) return e;
    *out = value;
    if (keeps) {
      std::lock_guard<std::mutex> lock(mutex_);
      if (!slots_[dev].ready.load(std::memory_order_relaxed)) {
        slots_[dev].value = value;
        slots_[dev].ready.store(true, std::memory_order_release);
      }
    }
    return E{};
  }

 private:
  static constexpr int kMost = 64;  // devices beyond are asked every time
  struct Slot {
    std::atomic<bool> ready{false};
    T value{};
  };
  Slot slots_[kMost];
  std::mutex mutex_;
};

}  // namespace ff
