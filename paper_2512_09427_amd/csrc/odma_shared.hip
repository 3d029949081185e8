// Entry point of decode attention over shared prefixes for gfx950: launches the kernels in shared_mfma.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "odma_internal.h"
#include "kernels_common.h"
#include "shared_mfma.h"
#include "device_common.h"

namespace {
// Heads of the batch beyond which a wave of the merge takes four: more waves than that are not on the chip at once.  1000 requests x 28
// heads behind 100 tokens 50.6 -> 46.5 us, 512 behind 200 47.9 -> 46.0; below it costs (128 x 28 behind 2048 38.0 -> 40.1).
constexpr int64_t SHARED_MANY = 8192;
// Heads up to which four waves share a head's pieces, of which there are most where few heads share the chip: 2 requests x 5 heads
// behind 30 623 tokens 25.2 -> 16.8 us, 1 x 28 behind 4096 15.5 -> 13.7, 1 x 1 with 30 000 of its own 29.4 -> 17.2, 4 x 28 behind 300 13.0 ->
// 13.1; above it costs more than it gives (16 x 28 behind 1000 15.8 -> 16.6, behind 16 384 25.6 -> 24.4).
constexpr int64_t SHARED_FEW = 128;
}  // namespace

extern "C" {

int odma_decode_attention_shared(odma_pool_t* pool, int32_t layer, int32_t n, const void* q, int32_t n_prefixes,
                                 const int32_t* prefix_start, const int64_t* prefix_offsets, const int32_t* prefix_lengths,
                                 const int64_t* offsets, const int32_t* lengths, const int32_t* block_table, int32_t bt_stride,
                                 void* out, void* stream) {
  const char* where = "odma_decode_attention_shared";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  const odma_pool_config_t& c = pool->cfg;
  auto refuse = [&](const char* why) {
    odma::set_error(std::string(where) + ": " + why);
    return ODMA_INVALID_ARG;
  };
  if (pool->decode_kernel != ODMA_KERNEL_MFMA) return refuse("needs a matrix-core pool (bf16 with head_dim 128 or 64, or fp8)");
  if (n == 0) return ODMA_OK;
  if (!c.workspace) return refuse("pool has no workspace");
  if (layer < 0 || layer >= c.n_layers || n < 0 || n > c.max_requests || !q || !lengths || !out || (!block_table && !offsets) ||
      (block_table && bt_stride <= 0))
    return refuse("invalid argument");
  if (n_prefixes < 0 || n_prefixes > n || (n_prefixes && (!prefix_start || !prefix_lengths || (!block_table && !prefix_offsets))))
    return refuse("0 to n prefixes, each with a start, an offset and a length");
  if (n_prefixes == 0) {
    rc = odma_decode_attention(pool, layer, n, q, offsets, lengths, block_table, bt_stride, out, 0, stream);
    pool->plan_stamp = {};                                     // (planned for lengths that no decode call has seen: not for reuse)
    return rc;
  }
  if (!(c.sm_scale > 0.f)) return refuse("needs a positive softmax scale");
  if (n > ODMA_SHARED_MAX_REQUESTS) return refuse("n exceeds ODMA_SHARED_MAX_REQUESTS");
  char* ws = (char*)c.workspace;
  const RowArgs ra = row_args(pool, layer);
  SharedArgs a;
  a.k = ra.k;
  a.v = ra.v;
  a.q = (const unsigned short*)q;
  a.out = out;
  a.prefix_start = prefix_start;
  a.prefix_lengths = prefix_lengths;
  a.prefix_offsets = prefix_offsets;
  a.offsets = offsets;
  a.lengths = lengths;
  a.bt = block_table;
  a.bt_stride = bt_stride;
  a.n = n;
  a.n_prefixes = n_prefixes;
  a.Hq = c.n_q_heads;
  a.Hkv = c.n_kv_heads;
  a.G = c.n_q_heads / c.n_kv_heads;
  a.head_stride = ra.head_stride;
  const bool fp8 = pool->elem_bytes == 1;
  a.scale_log2 = c.sm_scale * 1.4426950408889634f * (fp8 ? c.k_scale : 1.0f);
  a.out_scale = fp8 ? c.v_scale : 1.0f;
  a.out_bf16 = c.out_dtype == ODMA_BF16;
  // States live where the decode kernels keep theirs: 2 STREAM_MAX_WG columns per query head, the records of the requests
  // behind them.  First pieces take 2 columns per request and head; for each work-group there are the columns of a cut piece of line A and
  // of a group of heads for each of its waves: as many work-groups as that leaves room for, two per compute unit at most.
  const int64_t columns = (int64_t)2 * odma_plan::STREAM_MAX_WG * a.Hq;
  const int64_t rec_columns = ((int64_t)n * sizeof(SharedRecord) + sizeof(SharedShares) + 511) / 512;
  a.part_ml = (float2*)(ws + pool->ws.part_ml);
  a.part_o = (float*)(ws + pool->ws.part_o);
  a.rec = (SharedRecord*)(a.part_o + (columns - rec_columns) * 128);
  a.shares = (SharedShares*)(a.rec + n);
  a.cut_cols = (int32_t)std::min<int64_t>(SHARED_COLS, ((int64_t)n * a.G + 15) / 16 * 16);
  const int64_t room = (columns - rec_columns - (int64_t)2 * n * a.Hq) / (a.cut_cols + SHARED_WAVES * a.G);
  a.workers = (int32_t)std::min<int64_t>(2 * (int64_t)pool->n_cu, room) / 8 * 8;
  if (a.workers < 8) return refuse("too many requests for the partial results that the workspace holds");
  // The merge finds a state by its byte, in 32 bits, and its request by quotients below 2^20 (small_quotient).
  if ((int64_t)2 * n * a.Hq + (int64_t)a.workers * (a.cut_cols + SHARED_WAVES * a.G) >= 1 << 23 || (int64_t)n * a.Hkv >= 1 << 20)
    return refuse("too many heads for so many requests");
  hipStream_t s = (hipStream_t)stream;
  // [format][paged][fp32 results]
#define ODMA_SHARED(F) {{shared_parts_kernel<F, false, false>, shared_parts_kernel<F, false, true>}, {shared_parts_kernel<F, true, false>, shared_parts_kernel<F, true, true>}}
  static void (*const kernels[3][2][2])(SharedArgs) = {ODMA_SHARED(SHARED_BF16_128), ODMA_SHARED(SHARED_FP8_128), ODMA_SHARED(SHARED_BF16_64)};
  const int fmt = fp8 ? SHARED_FP8_128 : c.head_dim == 64 ? SHARED_BF16_64 : SHARED_BF16_128;
  hipLaunchKernelGGL(kernels[fmt][block_table != nullptr][!a.out_bf16], dim3(a.workers), dim3(SHARED_THREADS), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  const int64_t rows = (int64_t)n * a.Hq;
  const int kind = rows > SHARED_MANY ? 2 : rows <= SHARED_FEW ? 0 : 1;
  static void (*const merges[2][3])(SharedArgs) = {{shared_merge_kernel<128, 1, 4>, shared_merge_kernel<128, 1, 1>, shared_merge_kernel<128, 4, 1>},
                                                   {shared_merge_kernel<64, 1, 4>, shared_merge_kernel<64, 1, 1>, shared_merge_kernel<64, 4, 1>}};
  const int64_t waves = (int64_t)n * a.Hkv * (kind == 2 ? (a.G + 3) / 4 : a.G);
  hipLaunchKernelGGL(merges[c.head_dim == 64][kind], dim3((unsigned)(kind == 0 ? waves : (waves + 3) / 4)), dim3(256), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  return ODMA_OK;
}

}  // extern "C"
