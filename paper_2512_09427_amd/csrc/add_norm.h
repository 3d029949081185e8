// The residual stream between two blocks: the block's output is normed (if weights are given), gated and added, and the sum
// normed for the next block, in one pass over the row.
//
//   norm(x) = x / sqrt(mean(x^2) + eps)
//   r = residual_scale * residual + block_scale * gate * (block | norm(block) * block_weight),   x = norm(r) * next_weight
//
// Bound by memory: block, residual and gate are read once, the new residual and x written once; a row stays in registers from its
// loads to its stores.  A row's channels are dealt out to the lanes of W waves in pieces of eight.  65 869 rows of 3584 channels in bf16 beside
// a residual in fp32, both norms: 515 us, 5.5 TB/s (a copy of 1 GiB: 5.2); 256 rows 3.7 us, one row 2.2, which is a launch.
#pragma once

#include "kernels_common.h"
#include "row_pieces.h"
#include "wave_reduce.h"

namespace {

struct AddNormArgs {
  const void *block, *residual, *gate, *block_weight, *next_weight;
  const int64_t* row_slot;
  void *residual_out, *x_out;
  int64_t n_rows, pool_tokens;
  int64_t block_stride, residual_stride, gate_stride;    // elements between rows
  float eps, inv_width, residual_scale, block_scale;
  int32_t width, gate_kind;
};
constexpr float TINY = 0x1p-72f;     // the squares of 2^15 numbers up to 2^56 add up to less than fp32's largest

// T: rows; R: residual; W: waves of a row, P: pieces of eight channels a lane.  Work-groups of 256 threads, or of W waves where those
// are more.
template <typename T, typename R, int W, int P>
__global__ __launch_bounds__(W > 4 ? W * 64 : 256) void add_norm_kernel(AddNormArgs a) {
  constexpr int ROWS = W > 4 ? 1 : 4 / W;                  // rows of a work-group
  __shared__ float part[2][ROWS][W], again[2][ROWS][W];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int mine = W > 4 ? 0 : wave / W, w = W > 4 ? wave : wave % W;
  const int64_t row = (int64_t)blockIdx.x * ROWS + mine;
  bool there = row < a.n_rows;
  if (there && a.row_slot) {
    const int64_t slot = a.row_slot[row];
    there = slot != ODMA_SLOT_NONE && slot < a.pool_tokens;
  }
  if (W == 1 && !there) return;                            // (no barrier where a wave has a row of its own)
  constexpr bool EARLY = P <= 2;                           // weights too are loaded in the first round, where registers are plenty
  Piece<T> b[P], g[P], wb[P], wn[P];
  Piece<R> r[P];
  bool in[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int at = ((p * W + w) * 64 + lane) * 8;
    in[p] = there && at < a.width;
    b[p] = {};
    g[p] = {};
    r[p] = {};
    if (in[p]) {
      if (a.block) b[p] = take8((const T*)a.block + row * a.block_stride + at);
      r[p] = take8((const R*)a.residual + row * a.residual_stride + at);
      if (a.gate) g[p] = take8((const T*)a.gate + row * a.gate_stride + at);
      if (EARLY && a.block_weight) wb[p] = take8((const T*)a.block_weight + at);
      if (EARLY && a.next_weight) wn[p] = take8((const T*)a.next_weight + at);
    }
  }
  // 1 / sqrt(mean x^2 + eps) of a row in all its lanes; `turn`: those that follow one another take turns at two places.  A sum of squares beyond
  // fp32, whose mean may be within it, is formed again from smaller numbers, in which that of any finite row is (the branches cost 256 rows of 3584 channels
  // 0.1 us of 3.6).
  auto inverse_root = [&](auto x, int turn) {
    float ss = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = x(p, i);
        ss = __builtin_fmaf(v, v, ss);
      }
    float s = sum_over_wave(ss), small = 0.f;
    if (s == INFINITY) {                                     // (the whole wave)
      ss = 0.f;
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = x(p, i) * TINY;
          ss = __builtin_fmaf(v, v, ss);
        }
      small = sum_over_wave(ss);
    }
    if (W > 1) {
      if (lane == 0) {
        part[turn][mine][w] = s;
        if (s == INFINITY) again[turn][mine][w] = small;
      }
      __syncthreads();
      s = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) s += part[turn][mine][i];
      if (s == INFINITY) {
        small = 0.f;
#pragma unroll 1
        for (int i = 0; i < W; ++i) small += part[turn][mine][i] == INFINITY ? again[turn][mine][i] : part[turn][mine][i] * TINY * TINY;
      }
    }
    if (s == INFINITY) return root_of_inverse(__builtin_fmaf(small, a.inv_width, a.eps * TINY * TINY)) * TINY;
    return root_of_inverse(__builtin_fmaf(s, a.inv_width, a.eps));
  };
  float inv = 1.f;
  if (a.block_weight) {
    inv = inverse_root([&](int p, int i) {
      float x[8];
      widen8(b[p], x);
      return x[i];
    }, 0);
  }
  float v[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int at = ((p * W + w) * 64 + lane) * 8;
    float x[8], old[8];
    widen8(b[p], x);
    widen8(r[p], old);
    if (a.block_weight && in[p]) {
      float weight[8];
      widen8(EARLY ? wb[p] : take8((const T*)a.block_weight + at), weight);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * weight[i];
    }
    if (a.gate_kind != ODMA_GATE_NONE) {
      float gate[8];
      widen8(g[p], gate);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[i] *= a.gate_kind == ODMA_GATE_SIGMOID ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * gate[i])) : gate[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[p][i] = __builtin_fmaf(a.residual_scale, old[i], a.block_scale * x[i]);
    }
    if (a.residual_out && in[p]) put8((R*)a.residual_out + row * a.residual_stride + at, v[p]);
  }
  if (!a.x_out) return;
  inv = inverse_root([&](int p, int i) { return in[p] ? v[p][i] : 0.f; }, 1);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int at = ((p * W + w) * 64 + lane) * 8;
    if (!in[p]) continue;
    float weight[8];
    widen8(EARLY ? wn[p] : take8((const T*)a.next_weight + at), weight);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[p][i] = v[p][i] * inv * weight[i];
    put8((T*)a.x_out + row * a.width + at, v[p]);
  }
}

}  // namespace
