// Sums and maxima over the 64 lanes of a wave, in all of them: moves inside rows of 16 lanes (quads, then mirrors, which add the other half's
// equal results), and four reads for the four rows.  In the order of lanes' indices, always the same.
#pragma once

#include "kernels_common.h"

namespace {

template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ unsigned moved(unsigned x) {
  return (unsigned)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ float of_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
__device__ __forceinline__ unsigned of_lane(unsigned x, int lane) { return (unsigned)__builtin_amdgcn_readlane((int)x, lane); }

template <typename V, typename Op>
__device__ __forceinline__ V over_wave(V x, Op op) {
  x = op(x, moved<0xb1>(x));         // lanes 1 0 3 2
  x = op(x, moved<0x4e>(x));         // lanes 2 3 0 1
  x = op(x, moved<0x141>(x));        // halves of a row mirrored
  x = op(x, moved<0x140>(x));        // rows mirrored
  return op(op(of_lane(x, 0), of_lane(x, 16)), op(of_lane(x, 32), of_lane(x, 48)));
}
template <typename V>
__device__ __forceinline__ V sum_over_wave(V x) {
  return over_wave(x, [](V a, V b) { return a + b; });
}
__device__ __forceinline__ float max_over_wave(float x) {
  return over_wave(x, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace
