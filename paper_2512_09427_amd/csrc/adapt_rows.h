// Low-rank adapters of many requests beside a shared projection:
//   y[row, c] = base[row, c] + s_a sum_k up[a, c, k] h[row, k],   h[row, k] = sum_d down[a, k, d] x[row, d]
// for the rows of every item (adapter_lists.h: up to 64 rows of one adapter), in two launches, or in one where rows are few.
//
// The first of two forms h: ranks are the rows of the matrix product, an item's rows its columns.  The channels are cut between the waves of a
// work-group, which add up in LDS, and, where a batch has few items, between work-groups, whose parts stay apart in scratch: nothing is
// added up in an order that changes.  The second stages an item's h in LDS, parts added up and scaled, and takes 64 columns a wave at
// a time.  In bf16, h enters as three bf16 parts, which hold all its 24 bits: two of them side by side fill the contraction of 32 that a rank of 16 would
// half leave empty; from 24 ranks on one operand of up is multiplied by all three.  Two parts (16 bits of h) took 211 us and three take 213 for 43 340 rows of rank 16,
// 338 and 349 for rank 64, 123 and 137 for 8 326 rows of rank 128, but where base and products cancel the rest of a sum was that of 16 bits.
//
// Both are bound by memory: adapters that occur once are the bytes of a decode step, x, base and y those of a prompt.  3584 channels, 4608 columns, rank 16 in
// bf16: 43 340 rows of prompts 213 us (66 + 156 traced), 5.2 TB/s; 64 rows of as many adapters 11.4 us, a chain of loads that depend on one another (items, row
// numbers, x, columns) around 33 MB.  Larger ranks are not: 41 423 rows of rank 64 340 us (209 for the bytes), whose groups of ranks read x three times and whose
// weights come from the L2 for every item.  Large products in fp32 reach a ninth of the rate (0.154 PFLOP/s): 2 084 rows of rank 64, 1000 to 1024 channels, 22 us
// (5.1 for the bytes), one work-group on a compute unit, on 140 to 150 of them, with loads, 3.3 us of products, sums, loads and 3.4 us of products one behind the other.
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
  int32_t neighbours;                // first launch: items by fours (neighbours_of)
  int32_t runs;                      // the one launch for few rows: runs of 16 rows of the grid
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

// Which item a work-group has, of `pieces` each: eight items side by side, so that an item's work-groups share an XCD's L2.
__device__ __forceinline__ void item_of(int pieces, int& at, int& piece) {
  const int eight = blockIdx.x / (8 * pieces), rest = (int)blockIdx.x - eight * 8 * pieces;
  at = eight * 8 + rest % 8;
  piece = rest / 8;
}

// The same for many items: four neighbours, mostly of one adapter, share an XCD's L2 for their rows, which every group of ranks reads, and the ranks.
__device__ __forceinline__ void neighbours_of(int pieces, int& at, int& piece) {
  const int block = blockIdx.x / (32 * pieces), rest = (int)blockIdx.x - block * 32 * pieces, j = rest / 8;
  piece = j / 4;
  at = block * 32 + rest % 8 * 4 + j % 4;
}

// Rows that are more than a cache keeps pass by it.
template <bool STREAM, typename T>
__device__ __forceinline__ uint4v taken(const T* p) {
  return STREAM ? __builtin_nontemporal_load((const uint4v*)p) : *(const uint4v*)p;
}
template <bool STREAM, typename T>
__device__ __forceinline__ void put(T* p, uint4v v) {
  if (STREAM) __builtin_nontemporal_store(v, (uint4v*)p);
  else *(uint4v*)p = v;
}

// Eight ranks of h as the second product takes them in bf16: N numbers of 8 bits each, three or more, that add up to all 24 of h.  What is left of h is
// cut off, not rounded: finite numbers stay finite, what is left is exact, and all parts have h's sign.  Where nothing is left a part gives half of itself, so that
// none is 0 but of h of 0 (and of some below 2^-130), which beside an infinite weight would make a NaN of an infinity.
template <int N>
__device__ __forceinline__ void split_ranks(const float* v, uint4v (&part)[N]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float left[2] = {v[2 * e], v[2 * e + 1]};
#pragma unroll
    for (int q = 0; q < N; ++q) {
      unsigned bits[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float x = left[i], cut = __uint_as_float(__float_as_uint(x) & 0xffff0000u), half = 0.5f * x;
        const bool halved = q < N - 1 && cut == x;
        bits[i] = __float_as_uint(halved ? half : cut);
        left[i] = halved ? half : x - cut;
      }
      part[q][e] = bits[0] >> 16 | bits[1];
    }
  }
}

// A lane's part of a row's 64 columns: base and what the products add, rounded.  d: eight (fp32: four) sums.
__device__ __forceinline__ uint4v added(const unsigned short*, uint4v base, const float* d) {
  uint4v out;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    out[e] = float_to_bf16_bits(__uint_as_float(base[e] << 16) + d[2 * e]) | (unsigned)float_to_bf16_bits(__uint_as_float(base[e] & 0xffff0000u) + d[2 * e + 1]) << 16;
  return out;
}
__device__ __forceinline__ uint4v added(const float*, uint4v base, const float* d) {
  uint4v out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = __float_as_uint(__uint_as_float(base[e]) + d[e]);
  return out;
}

// h of an item: grid items x groups of MT tiles of 16 ranks x splits.
//
// A wave takes 128 bytes of the item's rows and of the ranks' at a time: lanes load them as they lie, eight neighbouring lanes a line, and
// pass them through LDS of the wave's own, where the pieces of a row are permuted by its number so that the 16 rows of an operand meet all banks.
template <typename T, int MT, bool STREAM>
__global__ __launch_bounds__(256) void adapt_down_kernel(AdaptArgs a) {
  using Op = AdaptOp<T>;
  constexpr int X = Op::X, CHUNK = 8 * X;                    // channels of a piece, of 128 bytes
  constexpr int WAVE = (64 + MT * 16) * 8;                   // pieces of a wave in LDS: rows, then ranks
  __shared__ __attribute__((aligned(16))) uint4v stage[4 * WAVE];
  int at = blockIdx.x / (a.splits * a.groups), cut = (int)blockIdx.x - at * a.splits * a.groups;
  if (a.neighbours) neighbours_of(a.splits * a.groups, at, cut);
  if (at >= a.max_items) return;
  const int4 item = a.items[at];
  const int adapter = item.x, first = item.y, count = min(item.z, ODMA_ADAPTER_ITEM_ROWS);
  if (count <= 0 || first < 0 || (unsigned)adapter >= (unsigned)a.n_adapters) return;
  const int lane = threadIdx.x & 63, wave = rfl(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int split = cut % a.splits, group = cut / a.splits;
  // the lane's line of eight, and which of its pieces it loads
  const int line = lane >> 3, piece = (lane & 7) ^ line;
  // the rows' numbers, in one round with the adapter's rank; rows that are not there repeat one: what they give is not used
  int number[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) number[i] = a.row_order[first + min(8 * i + line, count - 1)];
  const int flat = a.n_parts * a.rank, rank_a = rank_of(a, adapter);
  const int k0 = split * a.split_channels, k1 = min(k0 + a.split_channels, a.width);
  const int subtiles = (count + 15) / 16, r0 = group * MT * 16;
  uint4v* mine = stage + wave * WAVE;
  // ranks: eight at a time are all there or not (flat and the adapter's rank are multiples of 8); what those that are not hold is not used
  const T* arow = (const T*)a.down + ((int64_t)adapter * flat + r0 + line) * a.width + piece * X;
  bool there[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    const int r = r0 + 8 * i;
    there[i] = r < flat && r % a.rank < rank_a;
  }
  float4v acc[MT][4];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[t][u] = float4v{0.f, 0.f, 0.f, 0.f};
  auto run = [&](auto subs) {
    constexpr int NS = decltype(subs)::value;
    const T* xrow[2 * NS];
#pragma unroll
    for (int i = 0; i < 2 * NS; ++i) xrow[i] = (const T*)a.x + (number[i] >= 0 && number[i] < a.n_rows ? number[i] : 0) * a.x_stride + piece * X;
    uint4v av[2 * MT], xv[2 * NS];
    auto load = [&](int k) {
      const bool in = k + piece * X < k1;                    // (a width is whole pieces)
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) {
        av[i] = uint4v{0, 0, 0, 0};
        if (there[i] && in) av[i] = *(const uint4v*)(arow + (int64_t)(8 * i) * a.width + k);
      }
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) {
        xv[i] = uint4v{0, 0, 0, 0};
        if (in) xv[i] = taken<STREAM>(xrow[i] + k);
      }
    };
    int k = k0 + wave * CHUNK;
    if (k < k1) load(k);
    for (; k < k1; k += 4 * CHUNK) {
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) mine[i * 64 + lane] = xv[i];
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) mine[(8 + i) * 64 + lane] = av[i];
      if (k + 4 * CHUNK < k1) load(k + 4 * CHUNK);           // under way while these are multiplied
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint4v b[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u) b[u] = mine[(u * 16 + m) * 8 + ((4 * c + g) ^ (m & 7))];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const uint4v w = mine[(64 + t * 16 + m) * 8 + ((4 * c + g) ^ (m & 7))];
#pragma unroll
          for (int u = 0; u < NS; ++u) acc[t][u] = Op::mma(w, b[u], acc[t][u]);
        }
      }
    }
  };
  if (subtiles == 1) run(std::integral_constant<int, 1>{});
  else if (subtiles == 2) run(std::integral_constant<int, 2>{});
  else run(std::integral_constant<int, 4>{});
  // ---- the waves' sums; a lane holds ranks 4 g .. 4 g + 3 of row m
  float4v* parts = (float4v*)stage;
  float* out = a.h + ((int64_t)split * a.max_items + at) * ODMA_ADAPTER_ITEM_ROWS * flat;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (u >= subtiles) break;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t) parts[(wave * MT + t) * 64 + lane] = acc[t][u];
    __syncthreads();
    for (int t = wave; t < MT; t += 4) {
      const int r = r0 + t * 16 + 4 * g;
      if (r >= flat) continue;
      float4v s = parts[t * 64 + lane] + parts[(MT + t) * 64 + lane] + parts[(2 * MT + t) * 64 + lane] + parts[(3 * MT + t) * 64 + lane];
      if (r % a.rank >= rank_a) s = float4v{0.f, 0.f, 0.f, 0.f};
      *(float4v*)(out + (int64_t)(u * 16 + m) * flat + r) = s;
    }
  }
}

// Operands of h for 16 rows: in bf16 three parts of 32 ranks each, of up to 16 ranks four parts, two side by side in one; in fp32 16 ranks each.
template <typename T>
__host__ __device__ constexpr int up_steps(int rank) {
  return sizeof(T) == 4 ? (rank + 15) / 16 : rank <= 16 ? 2 : (rank + 31) / 32 * 3;
}
// Runs of 16 rows whose h is staged at a time, an operand of one 1 KiB, and the LDS for them.  Weights are read again for the next: 8 326 bf16 rows of rank 128 (12
// operands) 137 us with four runs, 166 with two; 8 326 fp32 rows of rank 160 (10) 525 and 608.
__host__ __device__ constexpr int up_staged(int steps) { return steps <= 12 ? 4 : steps <= 16 ? 2 : 1; }
constexpr size_t up_lds(int steps) { return (size_t)(steps <= 12 ? 4 * steps : 32) * 1024; }

// y of an item: grid items x chunks of columns.  SW: waves that share the rows of 64 columns where an item has so many.  LDS, dynamic: h in
// operand order, [subtile][step][group][row] pieces of 16 bytes.
//
// A tile of 16 rows x 64 columns leaves the accumulators through LDS of the wave's own and is added to base and stored as the rows lie,
// eight (fp32: 16) neighbouring lanes a line.
template <typename T, int SW, bool STREAM>
__global__ __launch_bounds__(256) void adapt_up_kernel(AdaptArgs a) {
  using Op = AdaptOp<T>;
  constexpr int X = Op::X, SUBS = 4 / SW;                    // most subtiles of a wave
  constexpr int LINE = 64 / X, LOADS = 16 * LINE / 64;       // lanes of a row's 64 columns; loads of a subtile
  extern __shared__ __attribute__((aligned(16))) uint4v hs[];
  __shared__ __attribute__((aligned(16))) float4v turned[4][256];
  const int at = blockIdx.x / a.chunks, chunk = (int)blockIdx.x - at * a.chunks;
  const int4 item = a.items[at];
  const int adapter = item.x, first = item.y, count = min(item.z, ODMA_ADAPTER_ITEM_ROWS);
  if (count <= 0 || first < 0 || (unsigned)adapter >= (unsigned)a.n_adapters) return;
  const int lane = threadIdx.x & 63, wave = rfl(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int flat = a.n_parts * a.rank, rank_a = rank_of(a, adapter);
  int part = 0;
  while (part + 1 < a.n_parts && chunk >= a.part_chunk[part + 1]) ++part;
  const int c0 = a.part_start[part] + (chunk - a.part_chunk[part]) * a.chunk_columns;
  const int c1 = min(c0 + a.chunk_columns, a.part_start[part + 1]), cols = a.part_start[a.n_parts];
  const bool narrow = X == 8 && a.rank <= 16;
  const int steps = up_steps<T>(a.rank), units = narrow ? 1 : X == 8 ? steps / 3 : steps;   // (units: operands of weights; in bf16 one serves all parts of h)
  const int eights = X == 8 && !narrow ? units * 4 : (a.rank + 15) / 16 * 2;                // of ranks
  const int line = lane / LINE, piece = lane % LINE;
  const float scale = a.scale ? a.scale[adapter] : 1.f;
  const T* up = (const T*)a.up + (int64_t)adapter * cols * a.rank;
  float4v* turn = turned[wave];
  const int most_rows = up_staged(steps) * 16;
  for (int j0 = 0; j0 < count; j0 += most_rows) {
    const int rows = min(count - j0, most_rows), subtiles = (rows + 15) / 16;
    // this wave's subtiles and columns
    const int sw = subtiles == 1 ? 1 : min(SW, subtiles == 3 ? 4 : subtiles), u0 = wave % sw, column_waves = 4 / sw;
    int row[SUBS][LOADS];
#pragma unroll
    for (int v = 0; v < SUBS; ++v)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) row[v][i] = a.row_order[first + j0 + min((u0 + v * sw) * 16 + i * (64 / LINE) + line, rows - 1)];
    uint4v in[SUBS][LOADS];
    auto load = [&](int cs) {
      const int c = cs + piece * X;
#pragma unroll
      for (int v = 0; v < SUBS; ++v)
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          if (row[v][i] >= 0 && c < c1) in[v][i] = taken<STREAM>((const T*)a.base + row[v][i] * a.base_stride + c);
    };
    auto piece_of = [&](int unit) { return narrow ? g & 1 : 4 * unit + g; };   // ranks of a lane's operand
    auto weights = [&](uint4v (&av)[4], int cs, int unit) {    // of 64 columns
      const int p = piece_of(unit);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int c = cs + t * 16 + m;
        av[t] = uint4v{0, 0, 0, 0};
        if (p * X < a.rank && c < c1) av[t] = *(const uint4v*)(up + (int64_t)c * a.rank + p * X);
      }
    };
    int cs = c0 + wave / sw * 64;
    uint4v av[4];
    if (cs < c1) weights(av, cs, 0);                           // under way while h is staged
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int v = 0; v < SUBS; ++v)
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        if ((u0 + v * sw) * 16 + i * (64 / LINE) + line >= rows || row[v][i] >= a.n_rows) row[v][i] = -1;
    if (cs < c1) load(cs);
    for (int i = threadIdx.x; i < subtiles * 16 * eights; i += 256) {
      const int j = i / eights, p = i - j * eights;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
      if (8 * p < a.rank && j < rows) {                      // (behind the adapter's rank h is 0)
        const float* src = a.h + ((int64_t)at * ODMA_ADAPTER_ITEM_ROWS + j0 + j) * flat + part * a.rank + 8 * p;
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
          const float* from = src + (int64_t)s * a.max_items * ODMA_ADAPTER_ITEM_ROWS * flat;
          const float4v lo = *(const float4v*)from, hi = *(const float4v*)(from + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] += lo[e];
            v[4 + e] += hi[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
      }
      uint4v* to = hs + (j >> 4) * steps * 64 + (j & 15);
      if constexpr (X == 8) {
        auto put_parts = [&](auto parts) {
          constexpr int N = decltype(parts)::value;
          uint4v h[N];
          split_ranks<N>(v, h);
#pragma unroll
          for (int q = 0; q < N; ++q) to[(q * eights + p) * 16] = h[q];
        };
        if (narrow) put_parts(std::integral_constant<int, 4>{});
        else put_parts(std::integral_constant<int, 3>{});
      } else {
        to[2 * p * 16] = __builtin_bit_cast(uint4v, float4v{v[0], v[1], v[2], v[3]});
        to[(2 * p + 1) * 16] = __builtin_bit_cast(uint4v, float4v{v[4], v[5], v[6], v[7]});
      }
    }
    __syncthreads();
    while (cs < c1) {
      float4v acc[SUBS][4];
#pragma unroll
      for (int v = 0; v < SUBS; ++v)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[v][t] = float4v{0.f, 0.f, 0.f, 0.f};
      for (int unit = 0; unit < units; ++unit) {
        if (unit > 0) weights(av, cs, unit);
        if (piece_of(unit) * X >= rank_a)                      // (what lies behind the adapter's rank may be anything)
#pragma unroll
          for (int t = 0; t < 4; ++t) av[t] = uint4v{0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < SUBS; ++v) {
          if (u0 + v * sw >= subtiles) break;
          const uint4v* b = hs + ((u0 + v * sw) * steps + unit) * 64 + lane;
#pragma unroll
          for (int t = 0; t < 4; ++t) acc[v][t] = Op::mma(av[t], b[0], acc[v][t]);
          if (X == 8) {
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[v][t] = Op::mma(av[t], b[units * 64], acc[v][t]);
            if (!narrow)
#pragma unroll
              for (int t = 0; t < 4; ++t) acc[v][t] = Op::mma(av[t], b[2 * units * 64], acc[v][t]);
          }
        }
      }
      const int now = cs + piece * X;
      cs += 64 * column_waves;
      uint4v old[SUBS][LOADS];
#pragma unroll
      for (int v = 0; v < SUBS; ++v)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) old[v][i] = in[v][i];
      if (cs < c1) {                                           // the next columns
        weights(av, cs, 0);
        load(cs);
      }
#pragma unroll
      for (int v = 0; v < SUBS; ++v) {
        if (u0 + v * sw >= subtiles) break;
        // a row's 16 pieces of four columns are permuted by its number
#pragma unroll
        for (int t = 0; t < 4; ++t) turn[m * 16 + ((4 * t + g) ^ m)] = acc[v][t];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int n = i * (64 / LINE) + line;
          float d[X];
#pragma unroll
          for (int e = 0; e < X / 4; ++e) {
            const float4v four = turn[n * 16 + ((piece * (X / 4) + e) ^ n)];
#pragma unroll
            for (int k = 0; k < 4; ++k) d[4 * e + k] = four[k];
          }
          const uint4v out = added((const T*)nullptr, old[v][i], d);
          if (row[v][i] >= 0 && now < c1) put<STREAM>((T*)a.y + row[v][i] * a.y_stride + now, out);
        }
      }
    }
    if (j0 + most_rows < count) __syncthreads();             // (h has been read)
  }
}

// Both products of 16 rows in one launch, for batches of few rows and ranks up to 64 (PT: tiles of 16): a work-group for every run of columns and 16 rows of an
// item, which forms what it needs of h for itself, from the caches where others do too.  Which 16 rows a work-group has it counts
// from all items (most have fewer than 16, and work-groups for rows that are not there would wait for a place all the same);
// eight of them stand side by side, so that those with the same rows are on one XCD.
template <typename T, int PT>
__global__ __launch_bounds__(512, PT == 1 ? 4 : 2) void adapt_few_kernel(AdaptArgs a) {
  using Op = AdaptOp<T>;
  constexpr int X = Op::X, CHUNK = 8 * X, WAVES = 8, AHEAD = PT == 4 ? 2 : 3;   // (AHEAD: runs of channels that a wave has under way)
  constexpr int LINE = 64 / X, LOADS = 16 * LINE / 64;
  constexpr int UNITS = X == 8 && PT > 1 ? PT / 2 : PT;      // operands of up and of h, as in the second of two launches
  constexpr int STEPS = X == 4 ? PT : PT == 1 ? 2 : 3 * UNITS;
  constexpr int TWO = PT < 2 ? PT : 2, WAVE = (16 + TWO * 16) * 8;   // of a wave in LDS: 16 rows and 16 or 32 ranks of 128 bytes, in pieces
  __shared__ __attribute__((aligned(16))) uint4v stage[WAVES * WAVE];
  __shared__ __attribute__((aligned(16))) uint4v hs[STEPS * 64];
  int run, chunk;
  item_of(a.chunks, run, chunk);
  const int wave = rfl(threadIdx.x >> 6);
  for (;; run += a.runs) {                                   // (lists of more rows than there are go on behind the grid's)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                           // (what follows from it is formed anew: nothing of it waits in registers for a second turn)
    const int m = lane & 15, g = lane >> 4;
    // ---- the run's item: 256 items a round
    int adapter = ODMA_ADAPTER_NONE, first = 0, count = 0, left = run;
    bool last = false;                                       // no run of the next round
    for (int i0 = 0; i0 < a.max_items && count == 0; i0 += 256) {
      int4 item[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        item[j] = make_int4(ODMA_ADAPTER_NONE, 0, 0, 0);
        if (i0 + j * 64 + lane < a.max_items) item[j] = a.items[i0 + j * 64 + lane];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int rows = (unsigned)item[j].x < (unsigned)a.n_adapters && item[j].y >= 0 ? min(max(item[j].z, 0), ODMA_ADAPTER_ITEM_ROWS) : 0;
        const int subs = (rows + 15) / 16;
        // runs of the items in front of this one (0 to 4 each), summed by their binary digits
        int before = 0, all = 0;
#pragma unroll
        for (int bit = 0; bit < 3; ++bit) {
          const unsigned long long set = __builtin_amdgcn_ballot_w64(subs >> bit & 1);
          before += (int)__builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0)) << bit;
          all += __builtin_popcountll(set) << bit;
        }
        if (count == 0 && left < all) {
          const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(left < before + subs));
          const int sub = left - __builtin_amdgcn_readlane(before, l);
          adapter = __builtin_amdgcn_readlane(item[j].x, l);
          first = __builtin_amdgcn_readlane(item[j].y, l) + sub * 16;
          count = min(__builtin_amdgcn_readlane(rows, l) - sub * 16, 16);
        }
        left -= all;
      }
      last = i0 + 256 >= a.max_items && left + a.runs >= 0;  // (left: this run behind all that there are)
    }
    if (count == 0) return;
    const int flat = a.n_parts * a.rank, rank_a = rank_of(a, adapter);
    int part = 0;
    while (part + 1 < a.n_parts && chunk >= a.part_chunk[part + 1]) ++part;
    const int c0 = a.part_start[part] + (chunk - a.part_chunk[part]) * a.chunk_columns;
    const int c1 = min(c0 + a.chunk_columns, a.part_start[part + 1]), cols = a.part_start[a.n_parts];
    uint4v* mine = stage + wave * WAVE;
    const int line8 = lane >> 3, piece8 = (lane & 7) ^ line8;
    const T* arow = (const T*)a.down + ((int64_t)adapter * flat + part * a.rank + line8) * a.width + piece8 * X;
    const int line = lane / LINE, piece = lane % LINE;
    // one round of loads for the rows' numbers, beside down and up; then x and base
    int xnumber[2], row[LOADS];
#pragma unroll
    for (int i = 0; i < 2; ++i) xnumber[i] = a.row_order[first + min(8 * i + line8, count - 1)];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) row[i] = a.row_order[first + min(i * (64 / LINE) + line, count - 1)];
    uint4v av[AHEAD][2 * PT], xv[AHEAD][2], in[LOADS], uv[UNITS][4];
    auto load_ranks = [&](int j, int k) {
      const bool there = k + piece8 * X < a.width;             // (a width is whole pieces)
#pragma unroll
      for (int i = 0; i < 2 * PT; ++i) {
        av[j][i] = uint4v{0, 0, 0, 0};
        if (8 * i < rank_a && there) av[j][i] = *(const uint4v*)(arow + (int64_t)(8 * i) * a.width + k);
      }
    };
    auto load_up = [&](int cs) {
#pragma unroll
      for (int s = 0; s < UNITS; ++s) {
        const int p = X == 8 && PT == 1 ? g & 1 : 4 * s + g;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uv[s][t] = uint4v{0, 0, 0, 0};
          if (p * X < rank_a && cs + t * 16 + m < c1) uv[s][t] = *(const uint4v*)((const T*)a.up + ((int64_t)adapter * cols + cs + t * 16 + m) * a.rank + p * X);
        }
      }
    };
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) load_ranks(j, (j * WAVES + wave) * CHUNK);
    int cs = c0 + wave * 64;
    if (PT == 1 && cs < c1) load_up(cs);
    __builtin_amdgcn_sched_barrier(0);
    const T* xrow[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) xrow[i] = (const T*)a.x + (xnumber[i] >= 0 && xnumber[i] < a.n_rows ? xnumber[i] : 0) * a.x_stride + piece8 * X;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      if (i * (64 / LINE) + line >= count || row[i] >= a.n_rows) row[i] = -1;
    auto load_x = [&](int j, int k) {
      const bool there = k + piece8 * X < a.width;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        xv[j][i] = uint4v{0, 0, 0, 0};
        if (8 * i < count && there) xv[j][i] = *(const uint4v*)(xrow[i] + k);
      }
    };
    auto load_base = [&](int cs) {
      const int c = cs + piece * X;
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        if (row[i] >= 0 && c < c1) in[i] = *(const uint4v*)((const T*)a.base + row[i] * a.base_stride + c);
    };
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) load_x(j, (j * WAVES + wave) * CHUNK);
    if (cs < c1) load_base(cs);
    const float scale = a.scale ? a.scale[adapter] : 1.f;
    float4v acc[PT];
#pragma unroll
    for (int t = 0; t < PT; ++t) acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
    for (int k = wave * CHUNK; k < a.width;) {
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (k >= a.width) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) mine[i * 64 + lane] = xv[j][i];
#pragma unroll
        for (int t0 = 0; t0 < PT; t0 += TWO) {
#pragma unroll
          for (int i = 0; i < 2 * TWO; ++i) mine[(2 + i) * 64 + lane] = av[j][2 * t0 + i];
          if (t0 + TWO >= PT && k + AHEAD * WAVES * CHUNK < a.width) {
            load_ranks(j, k + AHEAD * WAVES * CHUNK);
            load_x(j, k + AHEAD * WAVES * CHUNK);
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint4v b = mine[m * 8 + ((4 * c + g) ^ (m & 7))];
#pragma unroll
            for (int t = 0; t < TWO; ++t) acc[t0 + t] = Op::mma(mine[(16 + t * 16 + m) * 8 + ((4 * c + g) ^ (m & 7))], b, acc[t0 + t]);
          }
        }
        k += WAVES * CHUNK;
      }
    }
    // ---- the waves' sums, scaled, as the second product takes them; a lane holds ranks 4 g .. 4 g + 3 of row m
    float4v* parts = (float4v*)stage;
    if (PT > 1 && cs < c1) load_up(cs);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < PT; ++t) parts[(wave * PT + t) * 64 + lane] = acc[t];
    __syncthreads();
    if (wave < PT) {
      float4v sum = parts[wave * 64 + lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) sum += parts[(w * PT + wave) * 64 + lane];
      float v[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = 16 * wave + 4 * g < rank_a ? sum[e] * scale : 0.f;
        v[4 + e] = 0.f;
      }
      if constexpr (X == 8) {
        constexpr int PARTS = PT == 1 ? 4 : 3;
        uint4v h[PARTS];
        split_ranks<PARTS>(v, h);
        uint2v* to = (uint2v*)hs + ((2 * wave + (g >> 1)) * 16 + m) * 2 + (g & 1);
#pragma unroll
        for (int q = 0; q < PARTS; ++q) to[q * PT * 64] = uint2v{h[q][0], h[q][1]};
      } else {
        hs[(4 * wave + g) * 16 + m] = __builtin_bit_cast(uint4v, float4v{v[0], v[1], v[2], v[3]});
      }
    }
    __syncthreads();
    float4v* turn = (float4v*)mine;                            // (the parts have been read)
    while (cs < c1) {
      float4v sum[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        sum[t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) sum[t] = Op::mma(uv[s % UNITS][t], hs[s * 64 + lane], sum[t]);
      }
      uint4v old[LOADS];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) old[i] = in[i];
      const int now = cs + piece * X;
      cs += WAVES * 64;
      if (cs < c1) {
        load_up(cs);
        load_base(cs);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) turn[m * 16 + ((4 * t + g) ^ m)] = sum[t];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int n = i * (64 / LINE) + line;
        float d[X];
#pragma unroll
        for (int e = 0; e < X / 4; ++e) {
          const float4v four = turn[n * 16 + ((piece * (X / 4) + e) ^ n)];
#pragma unroll
          for (int k = 0; k < 4; ++k) d[4 * e + k] = four[k];
        }
        if (row[i] >= 0 && now < c1) *(uint4v*)((T*)a.y + row[i] * a.y_stride + now) = added((const T*)nullptr, old[i], d);
      }
    }
    if (last) return;
    __syncthreads();                                         // (LDS has been read)
  }
}

}  // namespace
