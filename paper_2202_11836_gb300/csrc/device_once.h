// Something that has to be done, or found out, once on every device (host code).
#pragma once
#include <atomic>
#include <cstdint>

namespace sky {

// Calls f for a device until it has returned 0 there once, and returns what it
// returned, else 0.  Threads may call it together (f may then run more than once).
class OncePerDevice {
 public:
  template <class F>
  auto operator()(int device, F&& f) -> decltype(f()) {
    // ordinals past the mask: every time
    const uint64_t bit = device >= 0 && device < 64 ? uint64_t{1} << device : 0;
    if (done_.load(std::memory_order_acquire) & bit) return decltype(f()){};
    const auto e = f();
    if (e == decltype(f()){}) done_.fetch_or(bit, std::memory_order_release);
    return e;
  }

 private:
  std::atomic<uint64_t> done_{0};
};

// A number of a device, such as how many clusters of a kernel it holds at once, that f finds out for it
// once.  What is not above 0 is a failure: it is returned and asked for again.  Threads may call it together.
class CountPerDevice {
 public:
  template <class F>
  int operator()(int device, F&& f) {
    const bool kept = device >= 0 && device < MOST;  // ordinals past them: every time
    if (kept)
      if (const int n = count_[device].load(std::memory_order_relaxed); n > 0) return n;
    const int n = f();
    if (kept && n > 0) count_[device].store(n, std::memory_order_relaxed);
    return n;
  }

 private:
  static constexpr int MOST = 64;
  std::atomic<int> count_[MOST] = {};
};

}  // namespace sky
