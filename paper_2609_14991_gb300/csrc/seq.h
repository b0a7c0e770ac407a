// Ragged rows: the sequence that holds a row of a call's row arrays.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace tsd {

// The sequence that holds a warp's row r: the last i with starts[i] <= r < starts[n]; -1: none
// (starts NULL: one row each).  Each round takes 32 probes at once.
__device__ __forceinline__ int seq_of(const int32_t* starts, int n, int r, int lane) {
  if (!starts) return r < n ? r : -1;
  int lo = 0, hi = n + 1;  // starts[lo] <= r < starts[hi], where both hold
  do {
    const int step = (hi - lo + 31) / 32, at = lo + step * lane;
    const unsigned below = __ballot_sync(0xffffffffu, at < hi && __ldg(starts + at) <= r);
    if (!below) return -1;
    lo += step * (31 - __clz(below));
    hi = min(lo + step, hi);
  } while (hi - lo > 1);
  return lo < n ? lo : -1;
}

}  // namespace tsd
