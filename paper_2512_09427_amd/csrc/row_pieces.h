// Eight neighbouring channels of a row, as they lie in memory and as numbers; what kernels that norm rows share.
#pragma once

#include "kernels_common.h"

namespace {

template <typename T>
struct Piece;
template <>
struct Piece<unsigned short> {
  uint4v w;
};
template <>
struct Piece<float> {
  float4v lo, hi;
};
__device__ __forceinline__ Piece<unsigned short> take8(const unsigned short* p) { return {*(const uint4v*)p}; }
__device__ __forceinline__ Piece<float> take8(const float* p) { return {*(const float4v*)p, *(const float4v*)(p + 4)}; }
__device__ __forceinline__ void widen8(const Piece<unsigned short>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.w[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen8(const Piece<float>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = r.lo[i];
    x[4 + i] = r.hi[i];
  }
}
__device__ __forceinline__ Piece<unsigned short> rounded8(const unsigned short*, const float* x) {
  uint4v w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (unsigned)float_to_bf16_bits(x[2 * i]) | ((unsigned)float_to_bf16_bits(x[2 * i + 1]) << 16);
  return {w};
}
__device__ __forceinline__ Piece<float> rounded8(const float*, const float* x) {
  return {float4v{x[0], x[1], x[2], x[3]}, float4v{x[4], x[5], x[6], x[7]}};
}
__device__ __forceinline__ void put8(unsigned short* p, const float* x) { *(uint4v*)p = rounded8(p, x).w; }
__device__ __forceinline__ void put8(float* p, const float* x) {
  const Piece<float> r = rounded8(p, x);
  *(float4v*)p = r.lo;
  *(float4v*)(p + 4) = r.hi;
}

// 1 / sqrt(v); the instruction takes denormal numbers for 0
__device__ __forceinline__ float root_of_inverse(float v) {
  const bool tiny = v < 0x1p-96f;
  return __builtin_amdgcn_rsqf(tiny ? v * 0x1p96f : v) * (tiny ? 0x1p48f : 1.f);
}

}  // namespace
