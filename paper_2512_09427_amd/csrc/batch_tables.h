// The tables of a batch: block tables, row starts and the slot of every new row, with prefixes that requests share.
#pragma once

#include "kernels_common.h"
#include "prefixes.h"

namespace {

struct TableArgs {
  const int32_t* lengths;        // [n]
  const int32_t* n_new;          // [n] or nullptr: one each
  const int64_t* offsets;        // [n]
  const int32_t* prefix_start;   // [n_prefixes + 1]
  const int64_t* prefix_offsets;
  const int32_t* prefix_lengths;
  int32_t n, n_prefixes, bt_stride;
  int32_t per;                   // requests of a work-group
  int32_t* block_table;          // [n][bt_stride] or nullptr
  int64_t max_rows;
  int64_t* row_start;            // [n + 1] or nullptr
  int32_t* row_position;         // [max_rows] or nullptr
  int64_t* row_slot;             // [max_rows] or nullptr
};

__device__ __forceinline__ int64_t wave_sum64(int64_t x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor((long long)x, o);
  return x;
}

// No arithmetic to speak of: a launch and the stores (64 requests, one new row each: 3.1 us; 256 prompts with 374 171 rows
// 5.3; 1024 requests with tables of 6.3 MB in all 4.8).  One work-group per request (or `per` of them beyond 1024 requests);
// blockIdx.y deals out the rows and entries of long ones.  Each finds its first row by adding up what all earlier requests
// bring, 256 of them a round, from the L2: a scan in a launch of its own would cost another launch, and a chained scan a
// round trip for every link.
__global__ __launch_bounds__(256) void build_tables_kernel(TableArgs a) {
  __shared__ int64_t part[4];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int r0 = blockIdx.x * a.per, r1 = min(r0 + a.per, a.n);
  const int step = 256 * gridDim.y, first = blockIdx.y * 256 + tid;
  auto new_rows = [&](int r) {
    const int len = max(a.lengths[r], 0);
    return a.n_new ? min(max(a.n_new[r], 0), len) : min(len, 1);
  };
  const bool rows = a.row_start || a.row_position || a.row_slot;
  int64_t at = 0;                                        // first row of the request
  if (rows) {
    for (int r = tid; r < r0; r += 256) at += new_rows(r);
    at = wave_sum64(at);
    if (lane == 0) part[wv] = at;
    __syncthreads();
    at = part[0] + part[1] + part[2] + part[3];
  }
  for (int r = r0; r < r1; ++r) {
    const int len = max(a.lengths[r], 0), p = a.n_prefixes ? prefix_of(a.prefix_start, a.n_prefixes, r) : -1;
    const int shared = p >= 0 ? shared_tokens(a.prefix_lengths[p]) : 0;
    const int64_t off = a.offsets[r];
    if (a.block_table) {
      const int blocks = (int)(((int64_t)len + BLK - 1) / BLK), in_prefix = shared / BLK;
      const int64_t pre = p >= 0 ? a.prefix_offsets[p] / BLK : 0, mine = off / BLK - in_prefix;
      int32_t* row = a.block_table + (int64_t)r * a.bt_stride;
      for (int64_t j = first; j < a.bt_stride; j += step)
        row[j] = j >= blocks ? 0 : (int32_t)((j < in_prefix ? pre : mine) + j);
    }
    if (rows) {
      const int count = new_rows(r), pos0 = len - count;
      if (a.row_start && first == 0) a.row_start[r] = at;
      if (a.row_position || a.row_slot) {
        const int64_t have = min((int64_t)count, a.max_rows - at);
        for (int64_t j = first; j < have; j += step) {
          const int pos = pos0 + (int)j;
          if (a.row_position) a.row_position[at + j] = pos;
          if (a.row_slot) a.row_slot[at + j] = pos < shared ? (int64_t)ODMA_SLOT_SHARED : off + (pos - shared);
        }
      }
      at += count;
    }
  }
  if (rows && r1 == a.n) {                               // the last request's work-groups: the total, and the rows behind it
    if (a.row_start && first == 0) a.row_start[a.n] = at;
    for (int64_t j = at + first; j < a.max_rows; j += step) {
      if (a.row_position) a.row_position[j] = 0;
      if (a.row_slot) a.row_slot[j] = ODMA_SLOT_NONE;
    }
  }
}

}  // namespace
