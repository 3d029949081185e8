// Entry points of libodma for gfx950 on a batch's rows around the attention: the residual stream (add_norm.h), rows by adapter
// (adapter_lists.h) and adapters beside a projection (adapt_rows.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "odma_internal.h"
#include "kernels_common.h"
#include "add_norm.h"
#include "adapter_lists.h"
#include "adapt_rows.h"
#include "device_common.h"

namespace {

int refuse(const char* where, const char* why) {
  odma::set_error(std::string(where) + ": " + why);
  return ODMA_INVALID_ARG;
}

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

constexpr int64_t MAX_ROWS = (int64_t)1 << 22;       // of odma_add_norm
constexpr int64_t MAX_THREADS = ((int64_t)1 << 32) - 1;   // of a launch
constexpr int64_t MAX_LISTED = (int64_t)1 << 27;     // rows of lists
constexpr int64_t MAX_WG = (1 << 24) - 1;            // work-groups of 256 threads of a launch
// Work-groups up to which the making of lists is dealt out, several requests each beyond: 1 024 requests of one row 6.7 us with 1 024 and 8.5 with 256, 2 048
// 12.7 with 1 024 and 17.4 with as many as requests; one of 8 192 rows 3.2 in eight work-groups and 5.3 in one.
constexpr int LIST_WG = 1024;

template <typename T, typename R, int W, int P>
void launch_add_norm(const AddNormArgs& a, hipStream_t s) {
  constexpr int rows = W > 4 ? 1 : 4 / W;
  hipLaunchKernelGGL((add_norm_kernel<T, R, W, P>), dim3((unsigned)((a.n_rows + rows - 1) / rows)), dim3(W > 4 ? W * 64 : 256), 0, s, a);
}

// Waves of a row and pieces of a lane: as many waves as a row fills with one piece a lane, more pieces from 16 waves on.  With many rows on
// a compute unit some widths take fewer waves with more pieces each, which wait for each other less.  us a call with few and with many waves: 3584
// channels 16 384 rows 83.3 (eight waves) and 87.5 (two), 65 869 beside an fp32 residual 526 and 515; 8 192 channels 256 rows 4.9 (16) and 5.0 (8), 1 024
// 13.0 and 11.6, 4 096 51 and 48.6; 520 channels 4 096 fp32 rows 7.6 (two) and 8.1 (one), 32 768 bf16 rows 32.3 and 29.6.  2 048 channels in one wave were
// slower throughout (4 096 rows 13.1 and 11.6 in four), in two the same as in four.  MAX_ROWS rows of 16 waves would be one thread more than a launch may have:
// they take eight waves.
constexpr int64_t NORM_MANY_2 = 64, NORM_MANY_8 = 192, NORM_MANY_16 = 4;   // rows a compute unit, by pieces
template <typename T, typename R>
void launch_add_norm(const AddNormArgs& a, int64_t n_cu, hipStream_t s) {
  const int pieces = (a.width + 511) / 512;                   // of 64 lanes
  if (pieces == 1) launch_add_norm<T, R, 1, 1>(a, s);
  else if (pieces == 2 && a.n_rows >= NORM_MANY_2 * n_cu) launch_add_norm<T, R, 1, 2>(a, s);
  else if (pieces == 2) launch_add_norm<T, R, 2, 1>(a, s);
  else if (pieces <= 4) launch_add_norm<T, R, 4, 1>(a, s);
  else if (pieces <= 8 && a.n_rows >= NORM_MANY_8 * n_cu) launch_add_norm<T, R, 2, 4>(a, s);
  else if (pieces <= 8) launch_add_norm<T, R, 8, 1>(a, s);
  else if (pieces <= 16 && a.n_rows >= NORM_MANY_16 * n_cu) launch_add_norm<T, R, 8, 2>(a, s);
  else if (pieces <= 16) launch_add_norm<T, R, 16, 1>(a, s);
  else if (a.n_rows * 1024 > MAX_THREADS) launch_add_norm<T, R, 8, 8>(a, s);
  else if (pieces <= 32) launch_add_norm<T, R, 16, 2>(a, s);
  else launch_add_norm<T, R, 16, 4>(a, s);
}

// Both products in one launch (adapt_few_kernel) or in two.  Every work-group of the one forms h for itself: its matrix instructions (counted as bytes of
// the ranks in bf16, in whole tiles of 16, four times as many for fp32) times the rounds of work-groups that the chip goes through must stay within what two launches
// cost more, which grows with the rows, and within a most.  One and two, us a call, 3584 channels, 4608 columns in three parts (1024 in one), requests of one row / adapters:
//   bf16, rank 16: 1 / 4 7.0 and 9.9, 64 / 64 11.7 and 16.8, 1 024 / 32 17.2 and 20.6, 4 096 / 32 43.2 and 44.9, 8 192 / 32 73 and 59.5
//   bf16, rank 32: 1 / 4 8.0 and 10.0, 256 / 32 17.6 and 18.1, 2 048 / 32 30.1 and 31.1, 4 096 / 32 56 and 52.7
//   bf16, rank 64: 1 / 4 12.6 and 10.5, 256 / 32 25.1 and 23.2 (13.8 and 17.2), 1 024 / 32 33.2 and 34.5 (14.9 and 19.9), 4 096 / 32 87 and 75 (32.9 and 32.3)
//   fp32, rank 64: 1 / 4 28.8 and 14.3, 256 / 32 59 and 46.5 (30 and 26.4), 1 024 / 32 78.5 and 90.5 (31.4 and 31.8), 4 096 / 32 180 and 192, 8 192 / 32 323 and 266
// other channels: bf16 208 / 3 of rank 64, 8 160 to 816 23.2 and 17.6; 15 / 15 of rank 64, 992 to 320 7.1 and 9.9; 4 132 / 32 of rank 16, 128 to 1072 10.0 and 16.8.
// (Figures below were taken when h had two parts in bf16; with three they are 1 to 4 % more on both sides.)
constexpr int64_t ADAPT_FEW = 8192, ADAPT_FEW_WORK = 320 << 10, ADAPT_FEW_ROW = 3 << 10, ADAPT_FEW_MOST = 560 << 10, ADAPT_FEW_MOST_F32 = 6 << 20, ADAPT_FEW_CU = 256;
// Work-groups that it is cut into, as far as the adapters that a batch may have let it be known.  Two share a compute unit with ranks up to 16: 64 / 64 as above
// 11.0 us with 260 and 12.3 with 390, 256 / 32 9.1 with 360 and 11.4 with 160.  With more it is one; parts narrower than the others' runs of columns
// leave short work-groups that fill in: fp32 1 024 / 32 of rank 64 77 us with 384 and 101 with 240, but beside 1024 columns 2 048 / 32 57 with 288 and 37 with 144.
constexpr int ADAPT_FEW_WG = 360, ADAPT_FEW_WG_PARTS = 400, ADAPT_FEW_WG_WIDE = 256;
// The first of two launches: fewest channels of a cut, and work-groups up to which channels are cut: every cut is one more array for the second
// launch to add up.  256 / 32 of rank 64 29.7 us with 512 and 32.8 with 256; 24 fp32 prompts of 2 300 rows 24.7 with 512 and 27.5 with 1024.
constexpr int ADAPT_SPLIT = 512, ADAPT_WG = 512;
// The second: work-groups up to which columns are cut, down to 64.  1 024 / 32 of rank 64 46 us with 1024 and 60 with 512.
constexpr int ADAPT_UP_WG = 1024;
// Two of its waves share the rows of 64 columns, four where a work-group has no more columns than that: 14 123 fp32 rows of 24 prompts
// beside 1024 columns 132 us with two and 153 with four.  Rows past the caches (shape.stream) where lines are whole, since two halves of a line that are
// stored one by one cross the memory twice: 93 308 rows of 80 + 2 000 columns, rank 64, 434 us past them and 324 through them, of 64 + 2 048 columns
// 263 and 277; 41 423 rows of 4 608 columns, rank 16, 219 and 245.
// ADAPT_UP_WG stands for long calls there too: work-groups of 512 columns.
// Of the first, groups of ranks of four neighbouring items on one XCD: 41 423 rows, three parts of rank 64, 332 us and 360 without.

// Runs of 16 rows of the items, as many as there can be if the lists are of these rows, in eights
inline int64_t few_runs(int64_t n_rows, int64_t items) { return (n_rows / 16 + std::min(items, n_rows) + 7) / 8 * 8; }

// Bytes of an element of the batch's rows: those of fp8 pools are bf16.
inline int row_bytes_of(const odma_pool_t* pool) { return pool->elem_bytes == 4 ? 4 : 2; }

// What the adapters' launches look like, or why they are refused.  n_rows < 0: for the scratch of any number of rows.
struct AdaptShape {
  int flat, tiles, groups, splits, split_channels, chunk_columns, chunks;
  bool few, stream, lines;
  size_t scratch;
};
const char* adapt_shape(const odma_adapters_t* ad, int row_bytes, int64_t n_rows, int64_t max_items, AdaptShape* shape) {
  if (!ad || !ad->down || !ad->up) return "adapters without weights";
  if (ad->n_adapters < 1 || ad->n_adapters > ODMA_MAX_ADAPTERS) return "1 to ODMA_MAX_ADAPTERS adapters";
  if (ad->rank < 8 || ad->rank > ODMA_MAX_RANK || ad->rank % 8) return "the rank must be a multiple of 8 up to ODMA_MAX_RANK";
  if (ad->width < 8 || ad->width % 8 || ad->width > ODMA_MAX_WIDTH) return "the width must be a multiple of 8 up to ODMA_MAX_WIDTH";
  if (ad->n_parts < 1 || ad->n_parts > ODMA_MAX_PARTS) return "1 to ODMA_MAX_PARTS parts";
  if (ad->part_start[0] != 0) return "the first part must start at column 0";
  for (int p = 0; p < ad->n_parts; ++p)
    if (ad->part_start[p + 1] <= ad->part_start[p] || ad->part_start[p + 1] % 16) return "parts must ascend by multiples of 16 columns";
  if (max_items < 0) return "invalid argument";
  if (!aligned(ad->down, 16) || !aligned(ad->up, 16)) return "weights must start on 16-byte boundaries";
  const int64_t items = std::max<int64_t>(max_items, 1);
  const int cols = ad->part_start[ad->n_parts];
  shape->flat = ad->n_parts * ad->rank;
  const int all = (shape->flat + 15) / 16;
  shape->tiles = std::min(all, 4);
  shape->groups = (all + shape->tiles - 1) / shape->tiles;
  shape->splits = (int)std::max<int64_t>(1, std::min<int64_t>((ad->width + ADAPT_SPLIT - 1) / ADAPT_SPLIT, ADAPT_WG / (items * shape->groups)));
  shape->split_channels = ((ad->width + shape->splits - 1) / shape->splits + 63) / 64 * 64;
  shape->splits = (ad->width + shape->split_channels - 1) / shape->split_channels;
  shape->scratch = std::max<size_t>((size_t)max_items * ODMA_ADAPTER_ITEM_ROWS * shape->flat * sizeof(float) * shape->splits, 256);
  auto chunks_of = [&](int columns) {
    int64_t n = 0;
    for (int p = 0; p < ad->n_parts; ++p) n += (ad->part_start[p + 1] - ad->part_start[p] + columns - 1) / columns;
    return n;
  };
  // One launch: its work-groups with the fewest chunks of columns that make enough of them, and how many rounds of them the chip goes through
  const int64_t listed = std::min(items, n_rows), least = n_rows / 16;
  const int64_t runs = ad->n_parts > 1 ? std::max(listed + n_rows / 64, least) : std::max(listed, least + (items - n_rows / 64) / 2);
  const int few_wg = ad->rank <= 16 ? ADAPT_FEW_WG : ad->n_parts > 1 ? ADAPT_FEW_WG_PARTS : ADAPT_FEW_WG_WIDE;
  int few_columns = 512;
  while (few_columns < 4096 && runs * chunks_of(few_columns) > few_wg) few_columns *= 2;
  const int64_t work = (int64_t)(ad->rank + 15) / 16 * 16 * ad->width * (row_bytes == 4 ? 8 : 2);
  const int64_t bound = std::min<int64_t>(ADAPT_FEW_WORK + ADAPT_FEW_ROW * n_rows, row_bytes == 4 ? ADAPT_FEW_MOST_F32 : ADAPT_FEW_MOST);
  shape->few = ad->rank <= 64 && n_rows >= 0 && n_rows <= ADAPT_FEW && items <= 1024 && cols <= 1 << 17 &&
               work * std::max<int64_t>(runs * chunks_of(few_columns), ADAPT_FEW_CU) <= bound * ADAPT_FEW_CU;
  shape->stream = n_rows * cols * row_bytes > (int64_t)4 << 20 && items * cols / 512 >= ADAPT_UP_WG;
  shape->chunk_columns = shape->few ? few_columns : 64;
  while (!shape->few && shape->chunk_columns < 512 && items * cols / shape->chunk_columns > ADAPT_UP_WG) shape->chunk_columns *= 2;
  if ((items + 31) / 32 * 32 * std::max<int64_t>(chunks_of(shape->chunk_columns), shape->splits * shape->groups) > MAX_WG) return "too many items";
  shape->chunks = (int)chunks_of(shape->chunk_columns);
  return nullptr;
}

template <typename T, bool STREAM>
void launch_adapt_down(const AdaptArgs& a, const AdaptShape& shape, hipStream_t s) {
  const dim3 grid((unsigned)(shape.splits * shape.groups * (a.neighbours ? (a.max_items + 31) / 32 * 32 : a.max_items)));
  if (shape.tiles == 1) hipLaunchKernelGGL((adapt_down_kernel<T, 1, STREAM>), grid, dim3(256), 0, s, a);
  else if (shape.tiles == 2) hipLaunchKernelGGL((adapt_down_kernel<T, 2, STREAM>), grid, dim3(256), 0, s, a);
  else if (shape.tiles == 3) hipLaunchKernelGGL((adapt_down_kernel<T, 3, STREAM>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((adapt_down_kernel<T, 4, STREAM>), grid, dim3(256), 0, s, a);
}

template <typename T>
int launch_adapt(const char* where, const AdaptArgs& a, const AdaptShape& shape, hipStream_t s) {
  hipError_t e;
  if (shape.few) {
    const dim3 grid((unsigned)(a.runs * shape.chunks));
    if (a.rank <= 16) hipLaunchKernelGGL((adapt_few_kernel<T, 1>), grid, dim3(512), 0, s, a);
    else if (a.rank <= 32) hipLaunchKernelGGL((adapt_few_kernel<T, 2>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((adapt_few_kernel<T, 4>), grid, dim3(512), 0, s, a);
    e = hipGetLastError();
    return e == hipSuccess ? ODMA_OK : hip_fail(where, e);
  }
  if (shape.stream && shape.groups == 1) launch_adapt_down<T, true>(a, shape, s);
  else launch_adapt_down<T, false>(a, shape, s);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  const dim3 grid((unsigned)(shape.chunks * a.max_items));
  const size_t lds = up_lds(up_steps<T>(a.rank));
  if (shape.stream && shape.lines) hipLaunchKernelGGL((adapt_up_kernel<T, 2, true>), grid, dim3(256), lds, s, a);
  else if (shape.chunk_columns > 64) hipLaunchKernelGGL((adapt_up_kernel<T, 2, false>), grid, dim3(256), lds, s, a);
  else hipLaunchKernelGGL((adapt_up_kernel<T, 4, false>), grid, dim3(256), lds, s, a);
  e = hipGetLastError();
  return e == hipSuccess ? ODMA_OK : hip_fail(where, e);
}

}  // namespace

extern "C" {

int odma_add_norm(odma_pool_t* pool, int64_t n_rows, const odma_add_norm_t* how, const void* block, int64_t block_stride,
                  const void* residual, int64_t residual_stride, const int64_t* row_slot, void* residual_out, void* x_out,
                  void* stream) {
  const char* where = "odma_add_norm";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  if (n_rows == 0) return ODMA_OK;
  if (n_rows < 0 || !how || !residual || (!residual_out && !x_out)) return refuse(where, "invalid argument");
  if (n_rows > MAX_ROWS) return refuse(where, "too many rows");
  if (how->width < 8 || how->width % 8 || how->width > ODMA_MAX_WIDTH) return refuse(where, "the width must be a multiple of 8 up to ODMA_MAX_WIDTH");
  const bool f32 = pool->elem_bytes == 4;
  if (how->residual_dtype != ODMA_F32 && (f32 || how->residual_dtype != ODMA_BF16))
    return refuse(where, "the residual has the rows' type or ODMA_F32");
  if (x_out && x_out == block && block_stride != how->width) return refuse(where, "x_out may be block only where block_stride is width");
  if (!x_out != !how->next_weight) return refuse(where, "x_out and next_weight go together");
  if (!block && (how->block_weight || how->gate)) return refuse(where, "weights or a gate without a block");
  if (how->gate_kind < ODMA_GATE_NONE || how->gate_kind > ODMA_GATE_SIGMOID || (how->gate_kind == ODMA_GATE_NONE) != !how->gate)
    return refuse(where, "gate and gate_kind do not go together");
  if (!(how->eps >= 0.f) || std::isinf(how->eps)) return refuse(where, "eps must be a finite number, 0 or more");
  if (!std::isfinite(how->residual_scale) || !std::isfinite(how->block_scale)) return refuse(where, "scales must be finite");
  const int unit = f32 ? 4 : 8, residual_unit = how->residual_dtype == ODMA_F32 ? 4 : 8;    // elements of 16 bytes
  if (!aligned(block, 16) || !aligned(residual, 16) || !aligned(residual_out, 16) || !aligned(x_out, 16) || !aligned(how->gate, 16) ||
      !aligned(how->block_weight, 16) || !aligned(how->next_weight, 16) || block_stride < 0 || block_stride % unit || residual_stride < 0 ||
      residual_stride % residual_unit || (how->gate && (how->gate_stride < 0 || how->gate_stride % unit)))
    return refuse(where, "rows and weights must start on 16-byte boundaries");
  if (residual_out && n_rows > 1 && residual_stride < how->width) return refuse(where, "rows of residual_out overlap");
  AddNormArgs a;
  a.block = block;
  a.residual = residual;
  a.gate = how->gate;
  a.block_weight = how->block_weight;
  a.next_weight = how->next_weight;
  a.row_slot = row_slot;
  a.residual_out = residual_out;
  a.x_out = x_out;
  a.n_rows = n_rows;
  a.pool_tokens = pool->pool_blocks * BLK;
  a.block_stride = block_stride;
  a.residual_stride = residual_stride;
  a.gate_stride = how->gate_stride;
  a.eps = how->eps;
  a.inv_width = 1.0f / (float)how->width;
  a.residual_scale = how->residual_scale;
  a.block_scale = how->block_scale;
  a.width = how->width;
  a.gate_kind = how->gate_kind;
  hipStream_t s = (hipStream_t)stream;
  if (f32) launch_add_norm<float, float>(a, pool->n_cu, s);
  else if (how->residual_dtype == ODMA_F32) launch_add_norm<unsigned short, float>(a, pool->n_cu, s);
  else launch_add_norm<unsigned short, unsigned short>(a, pool->n_cu, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  return ODMA_OK;
}

int odma_group_adapters(odma_pool_t* pool, int32_t n, const int32_t* adapter, int32_t n_adapters, const int64_t* row_start,
                        int64_t max_rows, int32_t* row_order, int32_t max_items, int32_t* items, void* stream) {
  const char* where = "odma_group_adapters";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  if (n < 0 || n > pool->cfg.max_requests || (n && !adapter) || max_rows < 0 || (max_rows && !row_order) || !items || !aligned(items, 16))
    return refuse(where, "invalid argument");
  if (n_adapters < 1 || n_adapters > ODMA_MAX_ADAPTERS) return refuse(where, "1 to ODMA_MAX_ADAPTERS adapters");
  if (max_rows > MAX_LISTED) return refuse(where, "too many rows");
  if (max_items < max_rows / ODMA_ADAPTER_ITEM_ROWS + std::min(n, n_adapters)) return refuse(where, "too few items for so many rows and adapters");
  ListArgs a;
  a.adapter = adapter;
  a.row_start = row_start;
  a.row_order = row_order;
  a.items = (int4*)items;
  a.max_rows = max_rows;
  a.n = n;
  a.n_adapters = n_adapters;
  a.max_items = max_items;
  a.per = std::max(1, (n + LIST_WG - 1) / LIST_WG);
  const int64_t wg = std::max(1, (n + a.per - 1) / a.per), longest = row_start ? max_rows / wg : 1;
  const int64_t split = std::max<int64_t>(1, std::min<int64_t>((longest + 1023) / 1024, LIST_WG / wg));
  const dim3 grid((unsigned)wg, (unsigned)split);
  const size_t lds = (size_t)(n_adapters + 31) / 32 * 4;
  if (row_start && n * max_rows > UINT32_MAX) hipLaunchKernelGGL((group_adapters_kernel<true>), grid, dim3(256), lds, (hipStream_t)stream, a);
  else hipLaunchKernelGGL((group_adapters_kernel<false>), grid, dim3(256), lds, (hipStream_t)stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  return ODMA_OK;
}

size_t odma_adapt_scratch_bytes(const odma_pool_t* pool, const odma_adapters_t* adapters, int32_t max_items) {
  const char* where = "odma_adapt_scratch_bytes";
  AdaptShape shape;
  const char* why = pool ? adapt_shape(adapters, row_bytes_of(pool), -1, max_items, &shape) : "null pool";
  if (why) {
    refuse(where, why);
    return 0;
  }
  return shape.scratch;
}

int odma_adapt_rows(odma_pool_t* pool, int64_t n_rows, const odma_adapters_t* adapters, int32_t max_items, const int32_t* items,
                    const int32_t* row_order, const void* x, int64_t x_stride, const void* base, int64_t base_stride, void* y,
                    int64_t y_stride, void* scratch, size_t scratch_bytes, void* stream) {
  const char* where = "odma_adapt_rows";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  if (n_rows == 0 || max_items == 0) return ODMA_OK;
  if (n_rows < 0 || !items || !row_order || !x || !base || !y || !scratch) return refuse(where, "invalid argument");
  if (n_rows > MAX_LISTED) return refuse(where, "too many rows");
  AdaptShape shape;
  const int row_bytes = row_bytes_of(pool);
  const char* why = adapt_shape(adapters, row_bytes, n_rows, max_items, &shape);
  if (why) return refuse(where, why);
  const int unit = 16 / row_bytes;                            // elements of 16 bytes
  if (!aligned(x, 16) || !aligned(base, 16) || !aligned(y, 16) || x_stride < 0 || x_stride % unit || base_stride < 0 || base_stride % unit ||
      y_stride < 0 || y_stride % unit)
    return refuse(where, "rows must start on 16-byte boundaries");
  const int32_t cols = adapters->part_start[adapters->n_parts];
  if (n_rows > 1 && y_stride < cols) return refuse(where, "rows of y overlap");
  if (y == base && y_stride != base_stride) return refuse(where, "y may be base only with the same stride");
  if (!aligned(items, 16) || !aligned(scratch, 256)) return refuse(where, "items must be 16-byte aligned, scratch 256-byte aligned");
  if (scratch_bytes < shape.scratch) return refuse(where, "scratch smaller than odma_adapt_scratch_bytes()");
  // whole lines of base and y in every work-group's columns
  shape.lines = aligned(base, 128) && aligned(y, 128) && base_stride * row_bytes % 128 == 0 && y_stride * row_bytes % 128 == 0;
  for (int p = 1; p < adapters->n_parts; ++p) shape.lines = shape.lines && adapters->part_start[p] * row_bytes % 128 == 0;
  AdaptArgs a;
  a.down = adapters->down;
  a.up = adapters->up;
  a.scale = adapters->scale;
  a.ranks = adapters->ranks;
  a.items = (const int4*)items;
  a.row_order = row_order;
  a.x = x;
  a.base = base;
  a.y = y;
  a.h = (float*)scratch;
  a.x_stride = x_stride;
  a.base_stride = base_stride;
  a.y_stride = y_stride;
  a.n_rows = n_rows;
  a.n_adapters = adapters->n_adapters;
  a.n_parts = adapters->n_parts;
  a.rank = adapters->rank;
  a.width = adapters->width;
  a.max_items = max_items;
  a.splits = shape.splits;
  a.split_channels = shape.split_channels;
  a.groups = shape.groups;
  a.chunk_columns = shape.chunk_columns;
  a.chunks = shape.chunks;
  a.neighbours = shape.stream && shape.groups > 1;
  a.runs = (int32_t)std::min<int64_t>(few_runs(n_rows, max_items), 1 << 20);
  for (int p = 0; p <= ODMA_MAX_PARTS; ++p) a.part_start[p] = p <= a.n_parts ? adapters->part_start[p] : cols;
  a.part_chunk[0] = 0;
  for (int p = 0; p < ODMA_MAX_PARTS; ++p)
    a.part_chunk[p + 1] = a.part_chunk[p] + (a.part_start[p + 1] - a.part_start[p] + a.chunk_columns - 1) / a.chunk_columns;
  hipStream_t s = (hipStream_t)stream;
  return row_bytes == 4 ? launch_adapt<float>(where, a, shape, s) : launch_adapt<unsigned short>(where, a, shape, s);
}

}  // extern "C"
