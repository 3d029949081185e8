// A batch's rows by adapter: the order of the rows, and items of up to 64 rows of one adapter (odma_group_adapters).
//
// A request's rows stand behind those of all requests with a smaller adapter, and of earlier ones with the same: two sums over
// the batch, which every request's work-group forms for itself, 256 requests a round, from the L2 -- a scan for all would be a launch of its
// own, or a chain.  Item numbers need no sum over adapters: that with `first` rows and d adapters in front of it begins at item first / 64 + d,
// behind the last item of the one before, since floor(f / 64) + ceil(c / 64) <= floor((f + c) / 64) + 1; d is a count over a bit map of
// the adapters that have rows.  Latency alone: loads, two barriers, stores.
#pragma once

#include "kernels_common.h"

namespace {

constexpr int ITEM_ROWS = ODMA_ADAPTER_ITEM_ROWS;

struct ListArgs {
  const int32_t* adapter;
  const int64_t* row_start;
  int32_t* row_order;
  int4* items;
  int64_t max_rows;
  int32_t n, n_adapters, max_items;
  int32_t per;                       // requests of a work-group
};

// LDS: the bit map, (n_adapters + 31) / 32 words.
__global__ __launch_bounds__(256) void group_adapters_kernel(ListArgs a) {
  extern __shared__ unsigned present[];
  __shared__ long long sums[4][4];
  __shared__ int counts[4][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = (a.n_adapters + 31) / 32;
  for (int i = tid; i < words; i += 256) present[i] = 0;
  __syncthreads();
  auto rows_of = [&](int s, int ad) -> long long {           // of a request with an adapter
    if (ad < 0 || ad >= a.n_adapters) return 0;
    if (!a.row_start) return 1;
    const long long rows = a.row_start[s + 1] - a.row_start[s];
    return rows < 0 ? 0 : rows < a.max_rows ? rows : a.max_rows;
  };
  long long all = 0;                                         // rows of the batch that have an adapter
  int distinct = 0;
  for (int i = 0; i < a.per; ++i) {
    const int r = blockIdx.x * a.per + i;
    if (r >= a.n && i > 0) break;
    const int mine = r < a.n ? a.adapter[r] : ODMA_ADAPTER_NONE;
    const bool has = mine >= 0 && mine < a.n_adapters;
    long long before = 0, first = 0, same = 0, total = 0;    // rows in front of the request's, of its adapter's, of its adapter, of all
    int earlier = 0;                                         // the adapter has rows of an earlier request
    for (int s = tid; s < a.n; s += 256) {
      const int ad = a.adapter[s];
      const long long rows = rows_of(s, ad);
      if (rows == 0) continue;
      if (i == 0) atomicOr(&present[ad >> 5], 1u << (ad & 31));
      total += rows;
      if (ad < mine) first += rows;
      if (ad == mine) same += rows;
      if (ad < mine || (ad == mine && s < r)) before += rows;
      if (ad == mine && s < r) earlier = 1;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      before += __shfl_xor(before, o);
      first += __shfl_xor(first, o);
      same += __shfl_xor(same, o);
      total += __shfl_xor(total, o);
      earlier |= __shfl_xor(earlier, o);
    }
    if (i > 0) __syncthreads();                              // (the sums of the request before have been read)
    if (lane == 0) {
      sums[wave][0] = before;
      sums[wave][1] = first;
      sums[wave][2] = same;
      sums[wave][3] = total;
      counts[wave][0] = earlier;
    }
    __syncthreads();
    before = sums[0][0] + sums[1][0] + sums[2][0] + sums[3][0];
    first = sums[0][1] + sums[1][1] + sums[2][1] + sums[3][1];
    same = sums[0][2] + sums[1][2] + sums[2][2] + sums[3][2];
    all = sums[0][3] + sums[1][3] + sums[2][3] + sums[3][3];
    earlier = counts[0][0] | counts[1][0] | counts[2][0] | counts[3][0];
    // adapters with rows: all of them, and those in front of this one (one number: both are at most 2^16)
    long long d = 0;
    for (int wd = tid; wd < words; wd += 256) {
      const unsigned bits = present[wd];
      d += (long long)__popc(bits) << 32;
      if (has) {
        if (wd < mine >> 5) d += __popc(bits);
        if (wd == mine >> 5) d += __popc(bits & ((1u << (mine & 31)) - 1u));
      }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) d += __shfl_xor(d, o);
    __syncthreads();                                         // (the sums have been read)
    if (lane == 0) sums[wave][0] = d;
    __syncthreads();
    d = sums[0][0] + sums[1][0] + sums[2][0] + sums[3][0];
    distinct = (int)(d >> 32);
    const int in_front = (int)(d & 0xffffffffll);
    const long long rows = has ? rows_of(r, mine) : 0;
    if (rows) {
      const long long from = a.row_start ? a.row_start[r] : r;
      for (long long j = blockIdx.y * 256 + tid; j < rows && before + j < a.max_rows; j += (long long)gridDim.y * 256)
        a.row_order[before + j] = (int32_t)(from + j);
      if (!earlier && blockIdx.y == 0) {                     // the adapter's items, and the one that may stay empty behind them
        const long long at = first / ITEM_ROWS + in_front, end = (first + same) / ITEM_ROWS + in_front + 1;
        for (long long j = tid; at + j < end && at + j < a.max_items; j += 256) {
          const long long f = first + j * ITEM_ROWS, left = (first + same < a.max_rows ? first + same : a.max_rows) - f;
          a.items[at + j] = left > 0 ? make_int4(mine, (int)f, (int)(left < ITEM_ROWS ? left : ITEM_ROWS), 0) : make_int4(ODMA_ADAPTER_NONE, 0, 0, 0);
        }
      }
    }
  }
  // behind the last adapter's
  const long long part = (long long)blockIdx.y * gridDim.x + blockIdx.x, parts = (long long)gridDim.x * gridDim.y;
  const long long used = distinct ? all / ITEM_ROWS + distinct : 0;
  for (long long j = used + part * 256 + tid; j < a.max_items; j += parts * 256) a.items[j] = make_int4(ODMA_ADAPTER_NONE, 0, 0, 0);
  for (long long j = all + part * 256 + tid; j < a.max_rows; j += parts * 256) a.row_order[j] = -1;
}

}  // namespace
