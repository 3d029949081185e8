// Entry points of libodma for gfx950 that prepare a batch: its tables (batch_tables.h) and its rows (qkv_rows.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "odma_internal.h"
#include "kernels_common.h"
#include "batch_tables.h"
#include "qkv_rows.h"
#include "device_common.h"

namespace {

int refuse(const char* where, const char* why) {
  odma::set_error(std::string(where) + ": " + why);
  return ODMA_INVALID_ARG;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T, typename S>
void launch_append_qkv(const QkvArgs& a, int group, dim3 grid, hipStream_t s) {
  if (group == 4) hipLaunchKernelGGL((append_qkv_kernel<T, S, 4>), grid, dim3(256), 0, s, a);
  else if (group == 8) hipLaunchKernelGGL((append_qkv_kernel<T, S, 8>), grid, dim3(256), 0, s, a);
  else if (group == 16) hipLaunchKernelGGL((append_qkv_kernel<T, S, 16>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((append_qkv_kernel<T, S, 32>), grid, dim3(256), 0, s, a);
}

constexpr int TABLES_WG = 1024;   // work-groups up to which a launch is dealt out
constexpr int ROWS_WG = 1024;     // (four a compute unit: a round of bf16 rows up to 128 channels and of fp8 pools; the kernels of fp32 rows and of bf16
                                  // rows beyond 128 channels hold 134 to 144 registers, three a compute unit, and a round is 768)
constexpr int64_t MAX_ROWS = (int64_t)1 << 27;   // (a launch has fewer than 2^32 threads)

}  // namespace

extern "C" {

int odma_build_tables(odma_pool_t* pool, int32_t n, const int32_t* lengths, const int32_t* n_new, const int64_t* offsets,
                      int32_t n_prefixes, const int32_t* prefix_start, const int64_t* prefix_offsets,
                      const int32_t* prefix_lengths, int32_t* block_table, int32_t bt_stride, int64_t max_rows,
                      int64_t* row_start, int32_t* row_position, int64_t* row_slot, void* stream) {
  const char* where = "odma_build_tables";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  if (n == 0) return ODMA_OK;
  if (n < 0 || n > pool->cfg.max_requests || !lengths || !offsets || (block_table && bt_stride <= 0) || max_rows < 0)
    return refuse(where, "invalid argument");
  if (n_prefixes < 0 || n_prefixes > n || (n_prefixes && (!prefix_start || !prefix_offsets || !prefix_lengths)))
    return refuse(where, "0 to n prefixes, each with a start, an offset and a length");
  if (!block_table && !row_start && !row_position && !row_slot) return refuse(where, "nothing to build");
  TableArgs a;
  a.lengths = lengths;
  a.n_new = n_new;
  a.offsets = offsets;
  a.prefix_start = prefix_start;
  a.prefix_offsets = prefix_offsets;
  a.prefix_lengths = prefix_lengths;
  a.n = n;
  a.n_prefixes = n_prefixes;
  a.bt_stride = block_table ? bt_stride : 0;
  a.per = (n + TABLES_WG - 1) / TABLES_WG;
  a.block_table = block_table;
  a.max_rows = row_position || row_slot ? max_rows : 0;
  a.row_start = row_start;
  a.row_position = row_position;
  a.row_slot = row_slot;
  const int64_t wg = (n + a.per - 1) / a.per, longest = std::max<int64_t>(a.max_rows / n, a.bt_stride);
  const int64_t split = std::min<int64_t>((longest + 1023) / 1024, std::max<int64_t>(TABLES_WG / wg, 1));
  hipLaunchKernelGGL(build_tables_kernel, dim3((unsigned)wg, (unsigned)std::max<int64_t>(split, 1)), dim3(256), 0, (hipStream_t)stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  return ODMA_OK;
}

int odma_append_qkv(odma_pool_t* pool, int32_t layer, int64_t n_rows, const odma_qk_prep_t* prep, const void* q,
                    int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                    const int64_t* row_slot, const int32_t* positions, void* q_out, void* stream) {
  const char* where = "odma_append_qkv";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  if (n_rows == 0) return ODMA_OK;
  const odma_pool_config_t& c = pool->cfg;
  if (layer < 0 || layer >= c.n_layers || n_rows < 0 || !prep || !q || !k || !v || !row_slot || !q_out)
    return refuse(where, "invalid argument");
  if (n_rows > MAX_ROWS) return refuse(where, "too many rows");
  const int unit = pool->elem_bytes == 4 ? 4 : 8;            // elements of 16 bytes of a row
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || q_stride < 0 || k_stride < 0 || v_stride < 0 ||
      q_stride % unit || k_stride % unit || v_stride % unit)
    return refuse(where, "rows must start on 16-byte boundaries");
  if (!aligned16(prep->q_weight) || !aligned16(prep->k_weight)) return refuse(where, "weights must start on 16-byte boundaries");
  if (!(prep->eps >= 0.f) || std::isinf(prep->eps)) return refuse(where, "eps must be a finite number, 0 or more");
  if (prep->rot_dim < 0 || prep->rot_dim > c.head_dim || prep->rot_dim % 8 || (prep->rot_dim && (!prep->inv_freq || !positions)))
    return refuse(where, "rot_dim must be a multiple of 8 up to head_dim, with frequencies and positions");
  if (prep->rot_pairs != ODMA_ROT_HALVES && prep->rot_pairs != ODMA_ROT_ADJACENT) return refuse(where, "unknown rot_pairs");
  if (prep->n_axes < 1 || prep->n_axes > ODMA_MAX_AXES) return refuse(where, "1 to ODMA_MAX_AXES axes");
  QkvArgs a;
  for (int f = 0; f < ODMA_MAX_ROT_PAIRS; ++f) {
    if (f < prep->rot_dim / 2 && prep->axis[f] >= prep->n_axes) return refuse(where, "a pair turns with an axis that is not there");
    a.axis[f] = prep->axis[f];
  }
  const RowArgs ra = row_args(pool, layer);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out = q_out;
  a.q_weight = prep->q_weight;
  a.k_weight = prep->k_weight;
  a.inv_freq = prep->inv_freq;
  a.row_slot = row_slot;
  a.positions = positions;
  a.n_rows = n_rows;
  a.pool_tokens = pool->pool_blocks * BLK;
  a.head_stride = ra.head_stride;
  a.k_pool = ra.k;
  a.v_pool = ra.v;
  a.eps = prep->eps;
  a.inv_D = 1.0f / (float)c.head_dim;
  a.k_inv = 1.0f / c.k_scale;
  a.v_inv = 1.0f / c.v_scale;
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.D = c.head_dim;
  a.rot_dim = prep->rot_dim;
  a.n_axes = prep->n_axes;
  a.adjacent = prep->rot_pairs == ODMA_ROT_ADJACENT;
  const int group = c.head_dim <= 32 ? 4 : c.head_dim <= 64 ? 8 : c.head_dim <= 128 ? 16 : 32;
  // Beyond an XCD's L2, queries leave past the caches and leave those to the keys and values, if a wave's store fills what it
  // touches (fp32 pairs in runs of four do not).  28 / 4 heads x 128, without and with it: 2 000 rows 14.0 -> 12.9 us,
  // 8 000 34.8 -> 31.5, 65 869 246 -> 244, not rotated 32.6 -> 26.2 at 8 000; fp32 rotated in halves 64.7 -> 63.2 at 8 000, and
  // 64.7 -> 67.7 not rotated, where it would touch halves of 32 bytes.
  a.stream_q = n_rows * a.Hq * a.D * (pool->elem_bytes == 4 ? 4 : 2) > (4 << 20) && (pool->elem_bytes != 4 || (!a.adjacent && a.rot_dim == a.D));
  // Multiples of ROWS_WG work-groups take 16 rows with all their heads each; the rows behind them (all, where there are few) deal
  // their heads out to about as many again, in whole batches or down to one pass of a work-group (28 / 4 heads x 128, whole batches
  // against any number of heads: 2 500 rows 14.7 -> 12.5 us, 3 000 16.8 -> 12.6, 10 000 41.9 -> 41.0).
  const int64_t tiles = (n_rows + BLK - 1) / BLK, whole = tiles / ROWS_WG * ROWS_WG, rest = tiles - whole;
  const int heads = a.Hq + 2 * a.Hkv, pass = rows_pass(group), batch = rows_batch(group, pool->elem_bytes), passes = (heads + pass - 1) / pass;
  const int split = rest ? (int)std::min<int64_t>(passes, (ROWS_WG + rest - 1) / rest) : 1;
  a.heads_per_wg = (passes + split - 1) / split * pass;
  if (a.heads_per_wg > batch) a.heads_per_wg = (a.heads_per_wg + batch - 1) / batch * batch;
  a.whole = (int32_t)whole;
  const int parts = (heads + a.heads_per_wg - 1) / a.heads_per_wg;
  a.rest = (int32_t)rest;
  a.rest_inverse = rest > 1 ? (uint32_t)(((1ull << 32) + rest - 1) / rest) : 0;   // (exact: rest * parts, at most 2 ROWS_WG, times rest is below 2^32)
  const dim3 grid((unsigned)(whole + rest * parts));
  hipStream_t s = (hipStream_t)stream;
  if (pool->elem_bytes == 1) hipLaunchKernelGGL((append_qkv_kernel<unsigned short, unsigned char, 16>), grid, dim3(256), 0, s, a);
  else if (pool->elem_bytes == 2) launch_append_qkv<unsigned short, unsigned short>(a, group, grid, s);
  else launch_append_qkv<float, float>(a, group, grid, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  return ODMA_OK;
}

}  // extern "C"
