// Prefixes that requests of a batch share: which request belongs to which, and how much is shared.
#pragma once

#include "kernels_common.h"

namespace {

// Group of request r: the last one that starts at or before it, if r lies before the next one's start; else -1.
__device__ __forceinline__ int prefix_of(const int32_t* start, int n_prefixes, int r) {
  int lo = 0, hi = n_prefixes + 1;                       // entries [0, lo) are <= r, entries [hi, ..) are not
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= r) lo = mid + 1;
    else hi = mid;
  }
  return lo >= 1 && lo <= n_prefixes ? lo - 1 : -1;
}
// the shared part of a prefix: its whole blocks
__device__ __forceinline__ int shared_tokens(int prefix_length) { return max(prefix_length, 0) / BLK * BLK; }

}  // namespace
