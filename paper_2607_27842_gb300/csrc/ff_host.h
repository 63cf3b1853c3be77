// Host-side helpers of the 8-bit layers that need no CUDA (tests compile them alone).
#pragma once

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

}  // namespace ff
