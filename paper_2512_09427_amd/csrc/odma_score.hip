// Entry point of token scores for gfx950: launches the kernels in score_tokens.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "odma_internal.h"
#include "kernels_common.h"
#include "score_tokens.h"
#include "device_common.h"

namespace {

int refuse(const char* where, const char* why) {
  odma::set_error(std::string(where) + ": " + why);
  return ODMA_INVALID_ARG;
}

constexpr int64_t MAX_ROWS = (int64_t)1 << 22;   // (a launch has fewer than 2^32 threads)
constexpr int32_t MAX_VOCAB = 1 << 24;
constexpr int PART_UNIT = 2048;       // elements of the shortest part: a piece or two for every thread of four waves

// Waves of a work-group and parts of a row: as many waves as a chip that has few rows can hold, in one work-group for each compute unit where
// there are about as many rows (16 waves), two (8), or more (4).  Rows of fewer tokens than SCORE_WHOLE stay whole, others are cut where
// rows are fewer than work-groups.  us a call, 20 alternatives, bf16: 256 rows x 128 000 22 with 16 waves, 27 with 8 or 16 in
// two parts, 33 with 4 in four; 300 x 128 000 33 (8), 36 (4); 512 x 128 000 34 (8), 41 (16), 45 (4); 8 rows x 128 000 11.5 in 63 parts of 4 waves, 12.3 of 8;
// whole against cut: 1 x 32 003 9.1 and 9.9, fp32 11.0 and 10.0; 100 x 32 003 10.5 and 13.5; 1 x 3 001 7.2 and 9.7; 1 x 65 003 12.4 and 9.9.
constexpr int SCORE_ROWS_4 = 512, SCORE_ROWS_8 = 256, SCORE_ROWS_16 = 16, SCORE_WHOLE = 32768;
constexpr int SCORE_WAVES = 4096;     // of a launch, where rows are cut

struct ScoreShape {
  int waves, parts, part_len;
  size_t states, scratch;
};
const char* score_shape(int64_t n_rows, int32_t vocab, int32_t n_top, ScoreShape* shape) {
  if (n_rows < 0 || n_rows > MAX_ROWS) return "too many rows";
  if (vocab < 1 || vocab > MAX_VOCAB) return "1 to 2^24 tokens";
  if (n_top < 0 || n_top > ODMA_MAX_ALTERNATIVES || n_top > vocab) return "0 to ODMA_MAX_ALTERNATIVES alternatives, of the vocabulary";
  const int64_t units = (vocab + PART_UNIT - 1) / PART_UNIT;
  const int64_t rows = std::max<int64_t>(n_rows, 1);
  const bool whole = vocab <= SCORE_WHOLE;
  shape->waves = rows > SCORE_ROWS_4 ? 4 : rows > SCORE_ROWS_8 ? 8 : rows >= SCORE_ROWS_16 || whole ? 16 : 4;
  const int64_t parts = whole ? 1 : std::max<int64_t>(1, std::min<int64_t>({units, SCORE_PARTS, SCORE_WAVES / shape->waves / rows}));
  shape->part_len = (int)((units + parts - 1) / parts * PART_UNIT);
  shape->parts = (vocab + shape->part_len - 1) / shape->part_len;
  shape->states = ((size_t)n_rows * shape->parts * sizeof(float4) + 255) / 256 * 256;
  shape->scratch = shape->parts == 1 ? 256 : std::max<size_t>(shape->states + (size_t)n_rows * shape->parts * n_top * sizeof(u64), 256);
  return nullptr;
}

template <typename T>
void launch_score(const ScoreArgs& a, int waves, dim3 grid, hipStream_t s) {
  if (waves == 4) hipLaunchKernelGGL((score_kernel<T, 4>), grid, dim3(256), 0, s, a);
  else if (waves == 8) hipLaunchKernelGGL((score_kernel<T, 8>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((score_kernel<T, 16>), grid, dim3(1024), 0, s, a);
}

}  // namespace

extern "C" {

size_t odma_score_scratch_bytes(const odma_pool_t* pool, int64_t n_rows, int32_t vocab, int32_t n_top) {
  ScoreShape shape;
  const char* why = pool ? score_shape(n_rows, vocab, n_top, &shape) : "null pool";
  if (!why) return shape.scratch;
  refuse("odma_score_scratch_bytes", why);
  return 0;
}

int odma_score_tokens(odma_pool_t* pool, int64_t n_rows, const void* logits, int64_t logits_stride, int32_t logits_dtype, int32_t vocab,
                      float scale, const int32_t* tokens, const int64_t* row_slot, int32_t n_top, float* logprob, int32_t* rank,
                      float* entropy, int32_t* top_id, float* top_logprob, void* scratch, size_t scratch_bytes, void* stream) {
  const char* where = "odma_score_tokens";
  int rc = device_ready(pool, where);
  if (rc) return rc;
  ScoreShape shape;
  const char* why = score_shape(n_rows, vocab, n_top, &shape);
  if (why) return refuse(where, why);
  if (n_rows == 0) return ODMA_OK;
  if (!logits || (logits_dtype != ODMA_F32 && logits_dtype != ODMA_BF16)) return refuse(where, "logits in ODMA_F32 or ODMA_BF16");
  if (logits_stride < 0 || (n_rows > 1 && logits_stride < vocab) || (uintptr_t)logits % (logits_dtype == ODMA_F32 ? 4 : 2))
    return refuse(where, "rows of logits overlap or are not aligned to their elements");
  if (!(scale >= 0x1p-24f && scale <= 0x1p24f)) return refuse(where, "the scale must lie between 2^-24 and 2^24");
  if (!tokens && (logprob || rank)) return refuse(where, "logprob and rank need tokens");
  if (!logprob && !rank && !entropy && !top_id && !top_logprob) return refuse(where, "nothing to compute");
  if (n_top == 0 && (top_id || top_logprob)) return refuse(where, "alternatives without their number");
  if (n_top && !top_id && !top_logprob) return refuse(where, "alternatives go nowhere");
  if (!scratch || (uintptr_t)scratch % 256 || scratch_bytes < shape.scratch)
    return refuse(where, "scratch of odma_score_scratch_bytes() bytes, 256-byte aligned");
  ScoreArgs a;
  a.logits = logits;
  a.logits_f32 = logits_dtype == ODMA_F32;
  a.stride = logits_stride;
  a.n_rows = n_rows;
  a.pool_tokens = pool->pool_blocks * BLK;
  a.tokens = tokens;
  a.row_slot = row_slot;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_logprob = top_logprob;
  a.rank = rank;
  a.top_id = top_id;
  a.part_state = (float4*)scratch;
  a.part_key = (u64*)((char*)scratch + shape.states);
  a.vocab = vocab;
  a.n_top = n_top;
  a.parts = shape.parts;
  a.part_len = shape.part_len;
  a.scale = scale;
  a.scale_log2 = scale * 1.4426950408889634f;
  int power;
  std::frexp(a.scale_log2, &power);
  a.far = std::ldexp(1.0f, SCORE_FAR_LOG2 - power);
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((unsigned)(n_rows * shape.parts));
  if (a.logits_f32) launch_score<float>(a, shape.waves, grid, s);
  else launch_score<unsigned short>(a, shape.waves, grid, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(where, e);
  if (shape.parts > 1) {
    hipLaunchKernelGGL(score_join_kernel, dim3((unsigned)n_rows), dim3(256), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(where, e);
  }
  return ODMA_OK;
}

}  // extern "C"
