// Where an element lies inside a block of the pools.
#pragma once

#include "kernels_common.h"

namespace {

// element index inside a block
__device__ __forceinline__ int k_index(int t, int d, int X) { return ((d / X) * BLK + t) * X + d % X; }
__device__ __forceinline__ int v_index(int t, int d) {
  return (((d >> 5) * 4 + (t >> 2)) * 16 + (d & 15)) * 8 + ((d >> 4) & 1) * 4 + (t & 3);
}
// fp8 storage (head_dim 128)
__device__ __forceinline__ int k_index_fp8(int t, int d) {
  return (((d >> 6) * 4 + ((d >> 3) & 3)) * 16 + t) * 16 + ((d >> 5) & 1) * 8 + (d & 7);
}
__device__ __forceinline__ int v_index_fp8(int t, int d) {
  return ((d >> 6) * 64 + (t >> 2) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (t & 3);
}

}  // namespace
