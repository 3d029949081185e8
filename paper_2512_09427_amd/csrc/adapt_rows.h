// Low-rank adapters of many requests beside a shared projection:
//   y[row, c] = base[row, c] + s_a sum_k up[a, c, k] h[row, k],   h[row, k] = sum_d down[a, k, d] x[row, d]
// for the rows of every item (adapter_lists.h: up to 64 rows of one adapter), two launches.
//
// The first forms h: ranks are the rows of the matrix product, an item's rows its columns, x and down come straight from
// memory in operand order (16 bytes a lane of both are neighbouring channels).  The channels are cut between the waves of a
// work-group, which add up in LDS, and, where a batch has few items, between work-groups, whose parts stay apart in scratch: nothing is
// added up in an order that changes.  The second stages an item's h in LDS, parts added up and scaled, and takes 64
// columns a wave at a time: base enters as the accumulators, y leaves as 16-byte pieces.  In bf16, h enters as two bf16 parts
// (value and rest: 16 bits), which fill the contraction of 32 that a rank of 16 would half leave empty.
//
// Both are bound by memory: adapters that occur once are the bytes of a decode step, x, base and y those of a prompt.
#pragma once

#include <type_traits>

#include "kernels_common.h"

namespace {

struct AdaptArgs {
  const void *down, *up;
  const float* scale;
  const int32_t* ranks;
  const int4* items;
  const int32_t* row_order;
  const void *x, *base;
  void* y;
  float* h;                          // [split][item][64 rows][all ranks]
  int64_t x_stride, base_stride, y_stride, n_rows;
  int32_t n_adapters, n_parts, rank, width, max_items;
  int32_t splits, groups, split_channels;   // first launch: cuts of the channels, of the ranks; channels of a cut
  int32_t part_start[ODMA_MAX_PARTS + 1];
  int32_t part_chunk[ODMA_MAX_PARTS + 1];   // second launch: chunks of columns in front of a part
  int32_t chunk_columns, chunks;
};

// An adapter's rank: a multiple of 8, up to that of the arrays.
__device__ __forceinline__ int rank_of(const AdaptArgs& a, int adapter) {
  if (!a.ranks) return a.rank;
  const int r = a.ranks[adapter];
  return r <= 0 ? 0 : r >= a.rank ? a.rank : (r + 7) & ~7;
}

// A 16-byte piece of each operand a lane: bf16 8 channels and one instruction; fp32 4 channels, an instruction for each.
template <typename T>
struct AdaptOp;
template <>
struct AdaptOp<unsigned short> {
  static constexpr int X = 8;
  static __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct AdaptOp<float> {
  static constexpr int X = 4;
  static __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    return c;
  }
};

// h of an item: grid items x groups of MT tiles of 16 ranks x splits.
template <typename T, int MT>
__global__ __launch_bounds__(256) void adapt_down_kernel(AdaptArgs a) {
  using Op = AdaptOp<T>;
  constexpr int X = Op::X, STEP = 4 * X, STEPS = 2;          // channels of a piece and of a step of four pieces; steps that a wave takes at a time
  __shared__ __attribute__((aligned(16))) float4v parts[4][MT][64];
  const int at = blockIdx.x / (a.splits * a.groups), cut = (int)blockIdx.x - at * a.splits * a.groups;
  const int4 item = a.items[at];
  const int adapter = item.x, first = item.y, count = min(item.z, ODMA_ADAPTER_ITEM_ROWS);
  if (count <= 0 || (unsigned)adapter >= (unsigned)a.n_adapters) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int split = cut % a.splits, group = cut / a.splits;
  const int flat = a.n_parts * a.rank, rank_a = rank_of(a, adapter);
  const int k0 = split * a.split_channels, k1 = min(k0 + a.split_channels, a.width);
  // ranks and rows that are not there repeat the first one: what they give is not used
  const T* arow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = (group * MT + t) * 16 + m;
    arow[t] = (const T*)a.down + ((int64_t)adapter * flat + (r < flat && r % a.rank < rank_a ? r : 0)) * a.width + g * X;
  }
  const int subtiles = (count + 15) / 16;
  const T* xrow[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int j = u * 16 + m;
    const int row = j < count ? a.row_order[first + j] : -1;
    xrow[u] = (const T*)a.x + (row >= 0 && row < a.n_rows ? row : 0) * a.x_stride + g * X;
  }
  float4v acc[MT][4];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[t][u] = float4v{0.f, 0.f, 0.f, 0.f};
  auto run = [&](auto subs) {
    constexpr int NS = decltype(subs)::value;
    for (int k = k0 + wave * STEPS * STEP; k < k1; k += 4 * STEPS * STEP) {
      uint4v av[STEPS][MT], xv[STEPS][NS];
#pragma unroll
      for (int c = 0; c < STEPS; ++c) {
        const bool in = k + c * STEP + g * X < k1;           // (a width is whole pieces)
#pragma unroll
        for (int t = 0; t < MT; ++t) av[c][t] = in ? *(const uint4v*)(arow[t] + k + c * STEP) : uint4v{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < NS; ++u) xv[c][u] = in ? *(const uint4v*)(xrow[u] + k + c * STEP) : uint4v{0, 0, 0, 0};
      }
#pragma unroll
      for (int c = 0; c < STEPS; ++c)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int u = 0; u < NS; ++u) acc[t][u] = Op::mma(av[c][t], xv[c][u], acc[t][u]);
    }
  };
  if (subtiles == 1) run(std::integral_constant<int, 1>{});
  else if (subtiles == 2) run(std::integral_constant<int, 2>{});
  else run(std::integral_constant<int, 4>{});
  // ---- the waves' sums; a lane holds ranks 4 g .. 4 g + 3 of row m
  float* out = a.h + ((int64_t)split * a.max_items + at) * ODMA_ADAPTER_ITEM_ROWS * flat;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (u >= subtiles) break;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t) parts[wave][t][lane] = acc[t][u];
    __syncthreads();
    for (int t = wave; t < MT; t += 4) {
      const int r = (group * MT + t) * 16 + 4 * g;
      if (r >= flat) continue;
      float4v s = parts[0][t][lane] + parts[1][t][lane] + parts[2][t][lane] + parts[3][t][lane];
      if (r % a.rank >= rank_a) s = float4v{0.f, 0.f, 0.f, 0.f};
      *(float4v*)(out + (int64_t)(u * 16 + m) * flat + r) = s;
    }
  }
}

// y of an item: grid items x chunks of columns.  LDS: h in operand order, [subtile][step][group][row] pieces of 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void adapt_up_kernel(AdaptArgs a) {
  using Op = AdaptOp<T>;
  constexpr int X = Op::X, NB = 16 / X;                      // pieces of a lane's 16 columns
  extern __shared__ __attribute__((aligned(16))) uint4v hs[];
  const int at = blockIdx.x / a.chunks, chunk = (int)blockIdx.x - at * a.chunks;
  const int4 item = a.items[at];
  const int adapter = item.x, first = item.y, count = min(item.z, ODMA_ADAPTER_ITEM_ROWS);
  if (count <= 0 || (unsigned)adapter >= (unsigned)a.n_adapters) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int flat = a.n_parts * a.rank, rank_a = rank_of(a, adapter);
  int part = 0;
  while (part + 1 < a.n_parts && chunk >= a.part_chunk[part + 1]) ++part;
  const int c0 = a.part_start[part] + (chunk - a.part_chunk[part]) * a.chunk_columns;
  const int c1 = min(c0 + a.chunk_columns, a.part_start[part + 1]), cols = a.part_start[a.n_parts];
  const int subtiles = (count + 15) / 16, steps = (a.rank + 15) / 16;
  int row[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int j = u * 16 + m;
    row[u] = j < count ? a.row_order[first + j] : -1;
    if (row[u] >= a.n_rows) row[u] = -1;
  }
  // ---- h: the splits' sums, scaled
  const float scale = a.scale ? a.scale[adapter] : 1.f;
  const int eights = steps * 2;                              // of ranks
  for (int i = threadIdx.x; i < subtiles * 16 * eights; i += 256) {
    const int j = i / eights, p = i - j * eights;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    if (8 * p < rank_a && j < count) {
      const float* src = a.h + ((int64_t)at * ODMA_ADAPTER_ITEM_ROWS + j) * flat + part * a.rank + 8 * p;
      for (int s = 0; s < a.splits; ++s) {
        const float4v lo = *(const float4v*)src, hi = *(const float4v*)(src + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] += lo[e];
          v[4 + e] += hi[e];
        }
        src += (int64_t)a.max_items * ODMA_ADAPTER_ITEM_ROWS * flat;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= scale;
    }
    uint4v* to = hs + (j >> 4) * steps * 64 + (j & 15);
    if constexpr (X == 8) {                                  // value and rest
      uint4v hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v0 = v[2 * e], v1 = v[2 * e + 1];
        const unsigned h0 = __float_as_uint(v0) & 0xffff0000u, h1 = __float_as_uint(v1) & 0xffff0000u;   // cut off: finite stays finite
        const float l0 = __builtin_isinf(v0) ? 0.f : v0 - __uint_as_float(h0), l1 = __builtin_isinf(v1) ? 0.f : v1 - __uint_as_float(h1);
        hi[e] = h0 >> 16 | h1;
        lo[e] = float_to_bf16_bits(l0) | (unsigned)float_to_bf16_bits(l1) << 16;
      }
      to[p * 16] = hi;
      to[(eights + p) * 16] = lo;
    } else {
      to[2 * p * 16] = __builtin_bit_cast(uint4v, float4v{v[0], v[1], v[2], v[3]});
      to[(2 * p + 1) * 16] = __builtin_bit_cast(uint4v, float4v{v[4], v[5], v[6], v[7]});
    }
  }
  __syncthreads();
  // ---- 64 columns a wave: four tiles whose rows are dealt out so that a lane's columns make pieces of 16 bytes, neighbouring lanes'
  // pieces 64
  for (int cs = c0 + wave * 64; cs < c1; cs += 256) {
    uint4v in[4][NB];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int c = cs + (b * 4 + g) * X;
        in[u][b] = row[u] >= 0 && c < c1 ? *(const uint4v*)((const T*)a.base + row[u] * a.base_stride + c) : uint4v{0, 0, 0, 0};
      }
    float4v acc[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (X == 8) {
            const unsigned w = in[u][t / 2][(t % 2) * 2 + i / 2];
            acc[u][t][i] = __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
          } else {
            acc[u][t][i] = __uint_as_float(in[u][t][i]);
          }
        }
    for (int s = 0; s < steps; ++s) {
      const int q = 4 * s + g, p = X == 8 && q >= eights ? q - eights : q;
      const bool real = p * X < rank_a;
      uint4v av[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int c = X == 8 ? cs + (t / 2) * 32 + (m / 4) * 8 + (t % 2) * 4 + m % 4 : cs + t * 16 + m;
        av[t] = real && c < c1 ? *(const uint4v*)((const T*)a.up + ((int64_t)adapter * cols + c) * a.rank + p * X) : uint4v{0, 0, 0, 0};
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (u >= subtiles) break;
        const uint4v bv = hs[(u * steps + s) * 64 + lane];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[u][t] = Op::mma(av[t], bv, acc[u][t]);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int c = cs + (b * 4 + g) * X;
        if (row[u] < 0 || c >= c1) continue;
        uint4v out;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (X == 8)
            out[i] = float_to_bf16_bits(acc[u][2 * b + i / 2][2 * (i % 2)]) | (unsigned)float_to_bf16_bits(acc[u][2 * b + i / 2][2 * (i % 2) + 1]) << 16;
          else
            out[i] = __float_as_uint(acc[u][b][i]);
        }
        *(uint4v*)((T*)a.y + row[u] * a.y_stride + c) = out;
      }
  }
}

}  // namespace
