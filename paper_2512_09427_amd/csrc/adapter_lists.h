// A batch's rows by adapter: the order of the rows, and items of up to 64 rows of one adapter (odma_group_adapters).
//
// A request's rows stand behind those of all requests with a smaller adapter, and of earlier ones with the same: two sums over
// the batch, which every request's work-group forms for itself, 256 requests a round, from the L2 -- a scan for all would be a launch of its
// own, or a chain.  Item numbers need no sum over adapters: that with `first` rows and d adapters in front of it begins at item first / 64 + d,
// behind the last item of the one before, since floor(f / 64) + ceil(c / 64) <= floor((f + c) / 64) + 1; d is a count over a bit map of
// the adapters that have rows.  Latency alone: loads, two barriers, stores; 256 requests of one row and 32 adapters 3.0 us, 512 prompts of 97 135 rows
// and 4 000 adapters 4.2.
#pragma once

#include "kernels_common.h"
#include "wave_reduce.h"

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

// LDS: the bit map, (n_adapters + 31) / 32 words.  CAPPED: for batches whose sums could be beyond 32 bits, which stay at max_rows (2^27 at most) once they are
// there; what is behind it does not exist.  256 requests of one row 3.00 us without and 3.09 with it, 512 prompts 4.13 and 4.31.
template <bool CAPPED>
__global__ __launch_bounds__(256) void group_adapters_kernel(ListArgs a) {
  extern __shared__ unsigned present[];
  __shared__ unsigned sums[2][4][6];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int words = (a.n_adapters + 31) / 32;
  for (int i = tid; i < words; i += 256) present[i] = 0;
  __syncthreads();
  auto rows_of = [&](int s, int ad) -> unsigned {            // of a request with an adapter
    if (ad < 0 || ad >= a.n_adapters) return 0;
    if (!a.row_start) return 1;
    const long long rows = a.row_start[s + 1] - a.row_start[s];
    return (unsigned)(rows < 0 ? 0 : rows < a.max_rows ? rows : a.max_rows);
  };
  const unsigned most = (unsigned)a.max_rows;
  auto plus = [&](unsigned x, unsigned y) { return CAPPED ? min(x + y, most) : x + y; };
  unsigned all = 0, distinct = 0;                            // rows of the batch that have an adapter, and adapters that have rows
  for (int i = 0; i < a.per; ++i) {
    const int r = blockIdx.x * a.per + i;
    if (r >= a.n && i > 0) break;
    const int mine = r < a.n ? a.adapter[r] : ODMA_ADAPTER_NONE;
    const bool has = mine >= 0 && mine < a.n_adapters;
    // rows in front of the request's, of its adapter's, of its adapter, of all; the adapter has rows of an earlier request
    unsigned before = 0, first = 0, same = 0, total = 0, earlier = 0;
    for (int s = tid; s < a.n; s += 256) {
      const int ad = a.adapter[s];
      const unsigned rows = rows_of(s, ad);
      if (rows == 0) continue;
      if (i == 0) atomicOr(&present[ad >> 5], 1u << (ad & 31));
      total = plus(total, rows);
      if (ad < mine) first = plus(first, rows);
      if (ad == mine) same = plus(same, rows);
      if (ad < mine || (ad == mine && s < r)) before = plus(before, rows);
      if (ad == mine && s < r) earlier = 1;
    }
    before = over_wave(before, plus);
    first = over_wave(first, plus);
    same = over_wave(same, plus);
    total = over_wave(total, plus);
    earlier = sum_over_wave(earlier);
    unsigned (*part)[6] = sums[i & 1];                       // (two sets: the one of the request before may still be read)
    if (lane == 0) {
      part[wave][0] = before;
      part[wave][1] = first;
      part[wave][2] = same;
      part[wave][3] = total;
      part[wave][4] = earlier;
    }
    __syncthreads();
    auto of_all = [&](int k) { return plus(plus(part[0][k], part[1][k]), plus(part[2][k], part[3][k])); };
    before = of_all(0);
    first = of_all(1);
    same = of_all(2);
    all = of_all(3);
    earlier = part[0][4] | part[1][4] | part[2][4] | part[3][4];
    // adapters with rows, all of them and those in front of this one: every wave counts for itself
    unsigned d = 0, in_front = 0;
    for (int wd = lane; wd < words; wd += 64) {
      const unsigned bits = present[wd];
      d += __popc(bits);
      if (has && wd <= mine >> 5) in_front += __popc(wd == mine >> 5 ? bits & ((1u << (mine & 31)) - 1u) : bits);
    }
    distinct = sum_over_wave(d);
    in_front = sum_over_wave(in_front);
    const unsigned rows = has ? rows_of(r, mine) : 0;
    if (rows) {
      const long long from = a.row_start ? a.row_start[r] : r;
      for (unsigned j = blockIdx.y * 256 + tid; j < rows && before + j < most; j += gridDim.y * 256)
        a.row_order[before + j] = from + j <= INT32_MAX ? (int32_t)(from + j) : -1;
      if (!earlier && blockIdx.y == 0) {                     // the adapter's items, and the one that may stay empty behind them
        const unsigned behind = plus(first, same), stop = min(behind, most);
        const unsigned at = first / ITEM_ROWS + in_front, end = behind / ITEM_ROWS + in_front + 1;
        for (unsigned j = tid; at + j < end && at + j < (unsigned)a.max_items; j += 256) {
          const unsigned f = first + j * ITEM_ROWS;
          a.items[at + j] = f < stop ? make_int4(mine, (int)f, (int)min(stop - f, (unsigned)ITEM_ROWS), 0) : make_int4(ODMA_ADAPTER_NONE, 0, 0, 0);
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
