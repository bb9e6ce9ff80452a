// Search in an ascending sequence by a whole warp.
#pragma once
#include <cuda_runtime.h>

namespace moe {

// The last i in [0, n) with key(i) <= at, or -1; key ascends.  By a whole warp, 32 candidates a step.
template <typename Key>
__device__ __forceinline__ int last_at_or_below(int n, long long at, int lane, Key key) {
  int lo = -1, hi = n;                                     // key(lo) <= at < key(hi)
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 31) / 32;
    const int i = lo + 1 + lane * step;
    const unsigned below = __ballot_sync(0xFFFFFFFFu, i < hi && key(i) <= at);
    const int found = 32 - __clz(below);                   // candidates at or below form a prefix
    const int base = lo;
    if (found > 0) lo = base + 1 + (found - 1) * step;
    hi = min(hi, base + 1 + found * step);
  }
  return lo;
}

}  // namespace moe
