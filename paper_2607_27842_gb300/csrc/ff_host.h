// Host-side helpers of the 8-bit layers that need no CUDA (tests compile them alone).
#pragma once

#include <atomic>
#include <mutex>

namespace ff {

// Calls f(first, n) for every run of at most `step` of `total` things, in order, until one
// returns something other than zero, and returns that.  64 bits: the step behind the last
// run of 2^31 - 256 things is past an int.
template <class F>
inline auto for_runs(long long total, long long step, F f) -> decltype(f(0ll, 0ll)) {
  using R = decltype(f(0ll, 0ll));
  for (long long at = 0; at < total; at += step) {
    const R r = f(at, total - at < step ? total - at : step);
    if (r != R(0)) return r;
  }
  return R(0);
}

// A value for each device, made by f(value) the first time the device is asked for; f
// returns zero, or an error that get() returns, and the next call tries again.  Calls of
// several threads make it once.
template <class T, int DEVICES = 64> class PerDevice {
  std::mutex m_;
  std::atomic<bool> made_[DEVICES] = {};
  T v_[DEVICES] = {};

 public:
  static constexpr int devices = DEVICES;
  template <class F> auto get(int device, T* out, F f) -> decltype(f(v_[0])) {
    using R = decltype(f(v_[0]));
    if (!made_[device].load(std::memory_order_acquire)) {
      std::lock_guard<std::mutex> lock(m_);
      if (!made_[device].load(std::memory_order_relaxed)) {
        const R r = f(v_[device]);
        if (r != R(0)) return r;
        made_[device].store(true, std::memory_order_release);
      }
    }
    *out = v_[device];
    return R(0);
  }
};

}  // namespace ff
