// Search by a whole wave.
#pragma once

#include <hip/hip_runtime.h>

namespace simsd {

// For how many b of [0, n) f(b) holds, where it holds for a leading part of them: 64
// probes a step, each the last b of its share.  (Uniform n; f is called by lanes whose
// probe is in range.)  4096 sequences take two round trips in place of 64 (a token each
// over 200 keys: attention 1321 -> 818 us, the cache append 34 -> 21).
template <typename F>
__device__ inline int leading(int n, int lane, F f) {
  int lo = 0, len = n;                           // f holds below lo, and not from lo + len on
  while (len > 0) {
    const int step = (len + 63) / 64;
    const int at = (lane + 1) * step - 1;
    const bool holds = at < len && f(lo + at);
    const int c = __popcll(__ballot(holds));
    lo += c * step;
    len = min(step - 1, len - c * step);
  }
  return lo;
}

}  // namespace simsd
