// Decode attention of a batch that shares prefixes, for gfx950.
//
// A request's softmax runs over its group's prefix and its own tokens.  Each of the two parts leaves a state of a query
// column (request, query head): reference m, sum l = sum 2^(s - m), O = sum 2^(s - m) V; states join by
//   M = max m_i,  out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i,
// so the prefix can be attended to by the queries of all its requests together: (requests x heads of a KV head's group)
// columns against its tokens, a dense contraction with reuse, where a request by itself only streams.
//
// Two lines of work.  Line A: items (prefix, KV head, block of SHARED_COLS columns), each the pairs of 16-token tiles of the
// prefix.  Line B: items (request, KV head), each the tiles of the request's own tokens.  Items are cut into chunks of tokens so
// that every work-group gets a like share of either line, and line A's matrix instructions run beside line B's memory traffic on
// every compute unit without a number that weighs one against the other: half of the work-groups begin with A, half with B.
// A chunk's piece leaves its state in the workspace and shared_merge_kernel joins them.  Line A is ordered (prefix, KV head,
// chunk, column block): the work-groups of an XCD read the same few chunks at a time, out of its L2.
#pragma once

#include "kernels_common.h"
#include "prefixes.h"

namespace {

typedef const int64_t __attribute__((address_space(4))) const_i64s;

enum { SHARED_BF16_128, SHARED_FP8_128, SHARED_BF16_64 };
constexpr int SHARED_COLS = 128;          // columns of an item of line A: four waves of two 16-column tiles
constexpr int SHARED_CT = 2;
constexpr int SHARED_A_EXTRA = 5;         // start and end of a piece of line A, in pairs
constexpr int SHARED_B_EXTRA = 8;         // and of line B, in tiles
constexpr int SHARED_A_LEAST = 8;         // pairs and tiles below which an item is not cut
constexpr int SHARED_B_LEAST = 12;
constexpr int SHARED_B_PIECES = 2;        // pieces of line B that a work-group gets on the average, where items are long enough
constexpr int SHARED_MAX_N = ODMA_SHARED_MAX_REQUESTS;
constexpr int SHARED_THREADS = 256;

struct SharedRecord {                     // of a request, for the merge
  int32_t a_chunks, a_blocks, a_col;      // line A: chunks (0: it shares nothing) and column blocks of an item, its first column
  int32_t a_extra;                        // cut pieces (chunks behind the first) in front of its group's
  int32_t b_chunks, b_extra;              // line B
  int32_t pad0, pad1;
};

struct SharedArgs {
  const char *k, *v;                      // layer base
  const unsigned short* q;
  void* out;
  const int32_t *prefix_start, *prefix_lengths;
  const int64_t *prefix_offsets, *offsets;
  const int32_t *lengths, *bt;
  int32_t bt_stride, n, n_prefixes, Hq, Hkv, G;
  int64_t head_stride;
  float scale_log2, out_scale;
  int32_t out_bf16;
  int32_t workers;                        // work-groups of the launch, a multiple of 8
  int32_t cut_cols;                       // columns kept for a cut piece of line A
  SharedRecord* rec;                      // [n]
  float2* part_ml;                        // states of columns: reference and sum
  float* part_o;                          // [column][128]
};

// Columns of the workspace: first chunks of line A and of line B by (request, head), then the chunks behind them, in the order of
// their line: at most `workers` of line A (SharedCut) and SHARED_B_PIECES times as many of line B.
__device__ __forceinline__ int64_t shared_first(const SharedArgs& a, int line, int r, int hq) {
  return ((int64_t)line * a.n + r) * a.Hq + hq;
}
__device__ __forceinline__ int64_t shared_cut_a(const SharedArgs& a, int i) { return (int64_t)2 * a.n * a.Hq + (int64_t)i * a.cut_cols; }
__device__ __forceinline__ int64_t shared_cut_b(const SharedArgs& a, int i) {
  return (int64_t)2 * a.n * a.Hq + (int64_t)a.workers * a.cut_cols + (int64_t)i * 16;
}

// How a line with `units` in `items` items is cut for `pieces` pieces in all: into chunks of at most `length`.  An item of T units
// has (T - 1) / length chunks behind its first, fewer than T / length, so all items together have fewer than units / length, which
// is at most `pieces` (half of them where items abound, so that they are cut little).
struct SharedCut {
  int length, shift;                                        // costs count 2^shift units, so that a line's sum fits 30 bits
  __device__ __forceinline__ SharedCut(float units, int items, int pieces, int least) {
    const float l = units * 1.0002f / (float)max(pieces - items, pieces / 2);   // (the sum is within 2^-13)
    length = max((int)fminf(l, 1e9f) + 1, least);
    shift = max(ilogbf(fmaxf(units, 1.f)) - 27, 0);
  }
  __device__ __forceinline__ int chunks(int T) const { return (T + length - 1) / length; }
};

// first unit of a chunk of an item of T units: chunks differ by one at most
__device__ __forceinline__ int chunk_start(int T, int chunks, int chunk) {
  const int base = T / chunks;
  return chunk * base + min(chunk, T - chunks * base);
}

// Work-group w takes the pieces of its share [start(w), start(w + 1)) of a line's cost.  The N pieces of an entry (a group, a request)
// that begins at s and costs c are spread over it evenly.
struct SharedShare {
  int x0, x1;
  __device__ __forceinline__ SharedShare(int total, int used, int w) {
    const double step = (double)total / (double)used;
    x0 = (int)((double)w * step);
    x1 = w + 1 >= used ? total : (int)((double)(w + 1) * step);
  }
  static __device__ __forceinline__ int upto(int x, int s, int c, int N) {
    return x <= s ? 0 : x >= s + c ? N : min((int)ceilf((float)(x - s) * (float)N / (float)c), N);   // (monotone in x)
  }
};

template <bool HIGH_HALF>
__device__ __forceinline__ unsigned widen_e4m3x2(unsigned w) {
  typedef float float2v __attribute__((ext_vector_type(2)));
  const float2v f = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HIGH_HALF);
  return (__float_as_uint(f[0]) >> 16) | (__float_as_uint(f[1]) & 0xffff0000u);
}

struct SharedPlan {
  int32_t a_pos[SHARED_MAX_N + 1], b_pos[SHARED_MAX_N + 1];   // cost in front of a group on line A, of a request on line B
  int32_t a_extra[SHARED_MAX_N], b_extra[SHARED_MAX_N];       // cut pieces in front of them
  int32_t start[SHARED_MAX_N + 1];                            // first request of a group
  int32_t tiles[SHARED_MAX_N];                                // of a group's shared part
  int32_t reader[SHARED_MAX_N];                               // of a group: its first request that holds all of the shared part
  int32_t own[SHARED_MAX_N];                                  // of a request: tokens that it reads itself
  int32_t skip[SHARED_MAX_N];                                 // ... and the blocks of its tokens in front of them (-1: in its group's prefix)
  float wave_units[SHARED_THREADS / 64];
  int32_t wave_items[SHARED_THREADS / 64];
  int32_t wave_sum[SHARED_THREADS / 64][4];
};

__device__ __forceinline__ int tiles_of(int tokens) { return (int)(((int64_t)tokens + BLK - 1) / BLK); }
__device__ __forceinline__ int column_blocks(int count, int G) { return (count * G + SHARED_COLS - 1) / SHARED_COLS; }

// Factor of a state joined to another.  At least the smallest number: 0 would make an infinite sum NaN.
__device__ __forceinline__ float joined(float m, float m_new) { return fmaxf(__builtin_amdgcn_exp2f(m - m_new), 0x1p-149f); }

// A weight as two bf16 parts: cut off, and the rest rounded (2^-16 in all).  Neither is negative, nor 0 unless the weight is: an
// infinite V times the parts is that infinity, as times the weight.
__device__ __forceinline__ void two_parts(float w, __bf16& hi, __bf16& lo) {
  const unsigned bits = __float_as_uint(w) & 0xffff0000u;
  hi = __builtin_bit_cast(__bf16, (unsigned short)(bits >> 16));
  lo = (__bf16)fmaxf(w - __uint_as_float(bits), w * 0x1p-40f);
}

// LO: the weights of line A go through the matrix cores as two bf16 parts (16 bits) instead of one; for fp32 results.
// (Line B, bound by memory, always does.)  A single rounding of a weight is half a bf16 step of one term of the sum, as the
// rounding of a bf16 result is of the whole.
template <int FMT, bool PAGED, bool LO>
__global__ __launch_bounds__(SHARED_THREADS, 2) void shared_parts_kernel(SharedArgs a) {
  constexpr bool FP8 = FMT == SHARED_FP8_128;
  constexpr int D = FMT == SHARED_BF16_64 ? 64 : 128;
  constexpr int NS = D / 32, DT = D / 16;                   // 32-channel steps, 16-channel groups
  constexpr int TILE_BYTES = BLK * D * (FP8 ? 1 : 2), LOADS = TILE_BYTES / 1024;
  constexpr int K_STAGE = 2 * NS * 1024, STAGE_BYTES = 2 * K_STAGE;
  constexpr int CT = SHARED_CT;
  constexpr float SLACK = 8.0f;                             // exponent units by which a score may exceed the reference
  constexpr int MERGE_BYTES = 4 * 16 * D * 4;               // line B: the waves' states
  __shared__ __attribute__((aligned(16))) char stage_mem[2 * STAGE_BYTES > MERGE_BYTES ? 2 * STAGE_BYTES : MERGE_BYTES];
  __shared__ float2 wave_ml[4][16];
  __shared__ SharedPlan plan;
  const int tid = threadIdx.x, lane = tid & 63, wv = rfl(tid >> 6);
  const int col16 = lane & 15, g4 = lane >> 4;
  const unsigned lane16 = lane * 16;
  const int G = a.G;

  // ---- plan: every work-group for itself (a launch of its own would be one work-group's round trips on an empty chip).  One
  // round of loads, then LDS alone.
  const int per = (a.n + SHARED_THREADS - 1) / SHARED_THREADS;
  const int r0 = min(tid * per, a.n), r1 = min(r0 + per, a.n);
  for (int r = tid; r < a.n; r += SHARED_THREADS) plan.own[r] = a.lengths[r];
  for (int p = tid; p <= a.n_prefixes; p += SHARED_THREADS) {
    plan.start[p] = min(max(a.prefix_start[p], 0), a.n);
    if (p < a.n_prefixes) {
      plan.tiles[p] = shared_tokens(a.prefix_lengths[p]) / BLK;
      plan.reader[p] = a.n;
    }
  }
  __syncthreads();
  float units = 0.f;
  int items = 0;
  for (int r = r0; r < r1; ++r) {
    const int len = max(plan.own[r], 0), p = prefix_of(plan.start, a.n_prefixes, r), shared = p >= 0 ? plan.tiles[p] * BLK : 0;
    const bool shares = shared > 0 && len >= shared;
    if (shares) atomicMin(&plan.reader[p], r);
    const int own = shares ? len - shared : len;
    plan.own[r] = own;
    plan.skip[r] = shares ? shared / BLK : shared > 0 ? -1 : 0;
    units += (float)tiles_of(own);
    items += own > 0;
  }
  units = wave_sum(units);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) items += __shfl_xor(items, o);
  if (lane == 0) {
    plan.wave_units[wv] = units;
    plan.wave_items[wv] = items;
  }
  __syncthreads();
  units = 0.f;
  items = 0;
  for (int i = 0; i < SHARED_THREADS / 64; ++i) {
    units += plan.wave_units[i];
    items += plan.wave_items[i];
  }
  const int b_items = items;
  const SharedCut cut_b(units * (float)a.Hkv, items * a.Hkv, SHARED_B_PIECES * a.workers, SHARED_B_LEAST);
  // groups, every wave for itself
  auto group_blocks = [&](int p) {                          // column blocks of a KV head; 0: nobody attends to the prefix
    return plan.reader[p] < a.n ? column_blocks(plan.start[p + 1] - plan.start[p], G) : 0;
  };
  units = 0.f;
  items = 0;
  for (int p = lane; p < a.n_prefixes; p += 64) {
    const int blocks = group_blocks(p);
    units += (float)blocks * (float)((plan.tiles[p] + 1) / 2);
    items += blocks;
  }
  units = wave_sum(units);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) items += __shfl_xor(items, o);
  const SharedCut cut_a(units * (float)a.Hkv, items * a.Hkv, a.workers, SHARED_A_LEAST);
  // costs and cut pieces, and their exclusive sums
  const int perp = (a.n_prefixes + SHARED_THREADS - 1) / SHARED_THREADS;
  const int p0 = min(tid * perp, a.n_prefixes), p1 = min(p0 + perp, a.n_prefixes);
  struct Entry {
    int cost, extra;
  };
  auto group_entry = [&](int p) {
    const int blocks = group_blocks(p), pairs = (plan.tiles[p] + 1) / 2, chunks = cut_a.chunks(pairs);
    if (!blocks) return Entry{0, 0};
    return Entry{(int)((int64_t)a.Hkv * blocks * (pairs + chunks * SHARED_A_EXTRA) >> cut_a.shift) + 1, a.Hkv * blocks * (chunks - 1)};
  };
  auto request_entry = [&](int r) {
    const int tiles = tiles_of(plan.own[r]), chunks = cut_b.chunks(tiles);
    if (!tiles) return Entry{0, 0};
    return Entry{(int)((int64_t)a.Hkv * (tiles + chunks * SHARED_B_EXTRA) >> cut_b.shift) + 1, a.Hkv * (chunks - 1)};
  };
  int sum[4] = {0, 0, 0, 0};
  for (int p = p0; p < p1; ++p) {
    const Entry e = group_entry(p);
    sum[0] += e.cost;
    sum[1] += e.extra;
  }
  for (int r = r0; r < r1; ++r) {
    const Entry e = request_entry(r);
    sum[2] += e.cost;
    sum[3] += e.extra;
  }
  int before[4], total[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) before[i] = sum[i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int y = __shfl_up(before[i], o);
      if (lane >= o) before[i] += y;
    }
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < 4; ++i) plan.wave_sum[wv][i] = before[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    before[i] -= sum[i];
    total[i] = 0;
    for (int w = 0; w < SHARED_THREADS / 64; ++w) {
      if (w < wv) before[i] += plan.wave_sum[w][i];
      total[i] += plan.wave_sum[w][i];
    }
  }
  for (int p = p0; p < p1; ++p) {
    const Entry e = group_entry(p);
    plan.a_pos[p] = before[0];
    plan.a_extra[p] = before[1];
    before[0] += e.cost;
    before[1] += e.extra;
  }
  for (int r = r0; r < r1; ++r) {
    const Entry e = request_entry(r);
    plan.b_pos[r] = before[2];
    plan.b_extra[r] = before[3];
    before[2] += e.cost;
    before[3] += e.extra;
  }
  if (tid == 0) {
    plan.a_pos[a.n_prefixes] = total[0];
    plan.b_pos[a.n] = total[2];
  }
  __syncthreads();
  if (blockIdx.x == gridDim.x - 1) {                        // for the merge
    for (int r = tid; r < a.n; r += SHARED_THREADS) {
      SharedRecord rec = {0, 0, 0, 0, cut_b.chunks(tiles_of(plan.own[r])), plan.b_extra[r], 0, 0};
      if (plan.skip[r] > 0) {
        const int p = prefix_of(plan.start, a.n_prefixes, r);
        rec.a_chunks = cut_a.chunks((plan.tiles[p] + 1) / 2);
        rec.a_blocks = group_blocks(p);
        rec.a_col = (r - plan.start[p]) * G;
        rec.a_extra = plan.a_extra[p];
      }
      a.rec[r] = rec;
    }
  }
  // XCD x (work-groups x, x + 8, ..) has neighbouring shares, which read the same heads.  A short line goes to few work-groups (a piece
  // each), the first ones of every XCD (A) or the last (B).
  auto used_of = [&](int cost, int pieces) { return cost ? min((min(pieces, a.workers) + 7) / 8 * 8, a.workers) : 0; };
  const int used_a = used_of(total[0], total[1] + items * a.Hkv), used_b = used_of(total[2], total[3] + b_items * a.Hkv);
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, turns = a.workers >> 3;
  const int ja = used_a >> 3, jb = used_b >> 3;
  const int share_a = turn < ja ? xcd * ja + turn : -1, share_b = turns - 1 - turn < jb ? xcd * jb + turns - 1 - turn : -1;

  auto piece = [&](const uint4v (&w)[LOADS], int s) {       // 16-byte operand s (of NS) of a tile, as bf16
    if (!FP8) return w[s % LOADS];
    const unsigned w0 = w[(s >> 1) % LOADS][2 * (s & 1)], w1 = w[(s >> 1) % LOADS][2 * (s & 1) + 1];
    return uint4v{widen_e4m3x2<false>(w0), widen_e4m3x2<true>(w0), widen_e4m3x2<false>(w1), widen_e4m3x2<true>(w1)};
  };
  auto join = [](uint2v lo, uint2v hi) { return __builtin_bit_cast(bf16x8, uint4v{lo[0], lo[1], hi[0], hi[1]}); };

  auto larger = [](float x, float y) { return __builtin_elementwise_maximum(x, y); };   // (NaN passes; fmaxf quiets every operand first)
  auto largest = [&](const float4v (&x)[2]) {
    return larger(larger(larger(x[0][0], x[0][1]), larger(x[0][2], x[0][3])), larger(larger(x[1][0], x[1][1]), larger(x[1][2], x[1][3])));
  };
  const float slack = SLACK / a.scale_log2;

  // ================= line A
  auto line_a = [&]() {
    bf16x8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;
    const SharedShare share(total[0], used_a, share_a);
    // group that holds x0: the last one at or before it (groups without work repeat a position)
    int lo = 0, hi = a.n_prefixes;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.a_pos[mid] <= share.x0) lo = mid;
      else hi = mid;
    }
    for (int p = rfl(lo); p < a.n_prefixes && plan.a_pos[p] < share.x1; ++p) {
      const int pos = rfl(plan.a_pos[p]), cost = rfl(plan.a_pos[p + 1]) - pos;
      if (!cost) continue;
      const int begin = rfl(plan.start[p]), count = rfl(plan.start[p + 1]) - begin;
      const int n_tiles = rfl(plan.tiles[p]), pairs = (n_tiles + 1) / 2, chunks = cut_a.chunks(pairs);
      const int blocks = column_blocks(count, G), per_head = chunks * blocks, n_pieces = a.Hkv * per_head, n_cols = count * G;
      const int64_t base_block = PAGED ? 0 : ((const const_i64s*)(uintptr_t)a.prefix_offsets)[p] / BLK;
      const const_i32* bt_row = as_constant(PAGED ? a.bt + (int64_t)rfl(plan.reader[p]) * a.bt_stride : nullptr);
      const int last = rfl(SharedShare::upto(share.x1, pos, cost, n_pieces));
      for (int id = rfl(SharedShare::upto(share.x0, pos, cost, n_pieces)); id < last; ++id) {
        const int g = rfl(id / per_head), chunk = rfl((id - g * per_head) / blocks), cb = id - g * per_head - chunk * blocks;
        const int i0 = rfl(chunk_start(pairs, chunks, chunk)), i1 = rfl(chunk_start(pairs, chunks, chunk + 1));
        const int cut = chunk ? rfl(plan.a_extra[p]) + (g * (chunks - 1) + chunk - 1) * blocks + cb : -1;
        const int c0 = cb * SHARED_COLS + wv * 16 * CT;
        const bool active = c0 < n_cols;
        const int64_t plane = (int64_t)g * a.head_stride;

        bool ok[CT];
        int row[CT], head[CT];
        bf16x8 qreg[CT][NS];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const int col = c0 + 16 * ct + col16;
          ok[ct] = col < n_cols;
          const int j = ok[ct] ? col / G : 0;
          row[ct] = begin + j;
          head[ct] = g * G + (ok[ct] ? col - j * G : 0);
          const unsigned short* qp = a.q + ((int64_t)row[ct] * a.Hq + head[ct]) * D + 8 * g4;
#pragma unroll
          for (int st = 0; st < NS; ++st) {
            const bf16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
            qreg[ct][st] = ok[ct] ? *(const bf16x8*)(qp + 32 * st) : z;
          }
        }
        // A column's reference m, in raw scores, enters with the accumulators of its scores (minus m instead of 0); -inf: none yet.
        // The sum of its weights is one more row of P V, with V = 1.
        float m[CT];
        float4v minus_m[CT], l[CT], O[CT][DT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          m[ct] = -INFINITY;
          minus_m[ct] = l[ct] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) O[ct][dt] = float4v{0.f, 0.f, 0.f, 0.f};
        }

        // loading: waves 0 and 1 bring K of the first and second tile of a pair, 2 and 3 V.  A second tile that does not exist
        // re-reads the first with its V zeroed (its scores are masked).
        const bool loads_v = wv >= 2;
        const int which = wv & 1;
        const char* src_base = (loads_v ? a.v : a.k) + plane;
        auto tile_of = [&](int pr) { return min(2 * min(pr, i1 - 1) + which, n_tiles - 1); };
        int blk_next = 0;
        auto lookup = [&](int pr) {
          if (PAGED) blk_next = bt_row[tile_of(pr)];
        };
        auto issue = [&](uint4v (&rg)[LOADS], int pr) {
          const char* src = src_base + (PAGED ? (int64_t)blk_next : base_block + tile_of(pr)) * TILE_BYTES;
#pragma unroll
          for (int i = 0; i < LOADS; ++i) rg[i] = *(const uint4v*)(src + i * 1024 + lane16);
        };
        auto write_stage = [&](const uint4v (&rg)[LOADS], int pr) {
          char* st = stage_mem + ((pr - i0) & 1) * STAGE_BYTES;
          const bool absent = 2 * min(pr, i1 - 1) + which >= n_tiles;
          if (!loads_v) {
            if (FP8) {
#pragma unroll
              for (int sp = 0; sp < NS; ++sp)
                *(uint4v*)(st + which * NS * 1024 + ((4 * sp + g4) * 16 + col16) * 16) = piece(rg, sp);
            } else {
#pragma unroll
              for (int i = 0; i < LOADS; ++i) *(uint4v*)(st + which * NS * 1024 + i * 1024 + lane16) = rg[i];
            }
          } else {
            char* dst = st + K_STAGE + lane16 + which * 8;
#pragma unroll
            for (int sp = 0; sp < NS; ++sp) {
              uint4v w = piece(rg, sp);
              if (absent) w = uint4v{0u, 0u, 0u, 0u};
              *(uint2v*)(dst + (2 * sp) * 1024) = uint2v{w[0], w[1]};
              *(uint2v*)(dst + (2 * sp + 1) * 1024) = uint2v{w[2], w[3]};
            }
          }
        };
        bool fresh = true;                                   // some column of the wave has no reference
        auto compute = [&](int pr) {
          const char* st = stage_mem + ((pr - i0) & 1) * STAGE_BYTES + lane16;
          bf16x8 av[DT];
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) av[dt] = *(const bf16x8*)(st + K_STAGE + dt * 1024);
          float4v x[CT][2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            bf16x8 kk[NS];
#pragma unroll
            for (int sp = 0; sp < NS; ++sp) kk[sp] = *(const bf16x8*)(st + b * NS * 1024 + sp * 1024);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
              float4v s4 = minus_m[ct];
#pragma unroll
              for (int sp = 0; sp < NS; ++sp) s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[sp], qreg[ct][sp], s4, 0, 0, 0);
              x[ct][b] = s4;
            }
          }
          if (2 * pr + 1 >= n_tiles) {
            asm volatile("");                                // (a branch: once an item, against eight selects a pair)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) x[ct][1] = float4v{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          }
          float top = -INFINITY;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) top = larger(top, largest(x[ct]));
          if (fresh || __builtin_amdgcn_ballot_w64(top > slack) != 0) {
            fresh = false;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
              float up = largest(x[ct]);
              up = fmaxf(up, __shfl_xor(up, 16));
              up = fmaxf(up, __shfl_xor(up, 32));
              float f = 1.f;
              if (m[ct] == -INFINITY) {
                m[ct] = up;
                up = up == -INFINITY ? 0.f : up;
              } else {
                up = fmaxf(up, 0.f);
                m[ct] += up;
                f = joined(0.f, up * a.scale_log2);
              }
              fresh |= __builtin_amdgcn_ballot_w64(m[ct] == -INFINITY) != 0;
              const float mm = m[ct] == -INFINITY ? 0.f : -m[ct];
              minus_m[ct] = float4v{mm, mm, mm, mm};
              l[ct] *= f;
#pragma unroll
              for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[ct][b][i] -= up;
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) O[ct][dt] *= f;
            }
          }
          bf16x8 ph[CT], pl[CT];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float pv = __builtin_amdgcn_exp2f(x[ct][b][i] * a.scale_log2);
                if (LO) {
                  __bf16 hi, lo;
                  two_parts(pv, hi, lo);
                  ph[ct][4 * b + i] = hi;
                  pl[ct][4 * b + i] = lo;
                } else {
                  ph[ct][4 * b + i] = (__bf16)pv;
                }
              }
            l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, ph[ct], l[ct], 0, 0, 0);
            if (LO) l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pl[ct], l[ct], 0, 0, 0);
          }
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
              O[ct][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], ph[ct], O[ct][dt], 0, 0, 0);
              if (LO) O[ct][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], pl[ct], O[ct][dt], 0, 0, 0);
            }
        };
        // pipeline: the loads of pair p + 2 are in flight while pair p is computed; pair p + 1 goes from registers into the
        // other stage behind it, and one barrier per pair makes it visible
        uint4v ra[LOADS], rb[LOADS];
        lookup(i0);
        issue(ra, i0);
        lookup(i0 + 1);
        issue(rb, i0 + 1);
        lookup(i0 + 2);
        __syncthreads();                                     // the stages of the piece before are done with
        write_stage(ra, i0);
        __syncthreads();
        auto step = [&](uint4v (&near)[LOADS], uint4v (&far)[LOADS], int pr) {
          issue(far, pr + 2);
          lookup(pr + 3);
          if (active) compute(pr);
          write_stage(near, pr + 1);
          __syncthreads();
        };
        for (int pr = i0;;) {
          step(rb, ra, pr);
          if (++pr == i1) break;
          step(ra, rb, pr);
          if (++pr == i1) break;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if (!ok[ct]) continue;
          const int64_t c = cut >= 0 ? shared_cut_a(a, cut) + wv * 16 * CT + 16 * ct + col16 : shared_first(a, 0, row[ct], head[ct]);
          if (g4 == 0) a.part_ml[c] = make_float2(m[ct] == -INFINITY ? LOWEST_REF : m[ct] * a.scale_log2, l[ct][0]);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) *(float4v*)(a.part_o + c * 128 + 16 * dt + 4 * g4) = O[ct][dt];
        }
      }
    }
  };

  // ================= line B: one request and KV head at a time; the waves take turns at its pairs of tiles, straight into registers
  auto line_b = [&]() {
    const SharedShare share(total[2], used_b, share_b);
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.b_pos[mid] <= share.x0) lo = mid;
      else hi = mid;
    }
    for (int r = rfl(lo); r < a.n && plan.b_pos[r] < share.x1; ++r) {
      const int pos = rfl(plan.b_pos[r]), cost = rfl(plan.b_pos[r + 1]) - pos;
      if (!cost) continue;
      const int own = rfl(plan.own[r]), tiles = tiles_of(own), chunks = cut_b.chunks(tiles), n_pieces = a.Hkv * chunks, skip = rfl(plan.skip[r]);
      // its own slab; a request shorter than the shared part reads its group's prefix
      int64_t base_block = 0;
      if (!PAGED)
        base_block = (skip >= 0 ? ((const const_i64s*)(uintptr_t)a.offsets)[r]
                                : ((const const_i64s*)(uintptr_t)a.prefix_offsets)[rfl(prefix_of(plan.start, a.n_prefixes, r))]) / BLK;
      const const_i32* bt_row = as_constant(PAGED ? a.bt + (int64_t)r * a.bt_stride + max(skip, 0) : nullptr);
      const int last = rfl(SharedShare::upto(share.x1, pos, cost, n_pieces));
      for (int id = rfl(SharedShare::upto(share.x0, pos, cost, n_pieces)); id < last; ++id) {
        const int g = rfl(id / chunks), chunk = id - g * chunks;
        const int i0 = rfl(chunk_start(tiles, chunks, chunk)), i1 = rfl(chunk_start(tiles, chunks, chunk + 1));
        const int cut = chunk ? rfl(plan.b_extra[r]) + g * (chunks - 1) + chunk - 1 : -1;
        const int64_t plane = (int64_t)g * a.head_stride;
        bf16x8 qreg[NS];
        {
          const unsigned short* qp = a.q + ((int64_t)r * a.Hq + g * G + min(col16, G - 1)) * D + 8 * g4;
#pragma unroll
          for (int st = 0; st < NS; ++st) {
            const bf16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
            qreg[st] = col16 < G ? *(const bf16x8*)(qp + 32 * st) : z;
          }
        }
        float m = LOWEST_REF, l = 0.f;
        float4v O[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[dt] = float4v{0.f, 0.f, 0.f, 0.f};
        uint4v kr[2][LOADS], vr[2][LOADS];
        auto at_of = [&](int t, int b) {
          const int tile = min(t + b, i1 - 1);
          return plane + (PAGED ? (int64_t)bt_row[tile] : base_block + tile) * TILE_BYTES;
        };
        auto load = [&](uint4v (&to)[2][LOADS], const char* pool, int t) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const char* src = pool + at_of(t, b) + lane16;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) to[b][i] = __builtin_nontemporal_load((const uint4v*)(src + i * 1024));
          }
        };
        const int first = i0 + 2 * wv;
        if (first < i1) {
          load(kr, a.k, first);
          load(vr, a.v, first);
        }
        for (int t = first; t < i1; t += 8) {
          const bool more = t + 8 < i1;
          float4v x[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            float4v s4 = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int sp = 0; sp < NS; ++sp)
              s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, piece(kr[b], sp)), qreg[sp], s4, 0, 0, 0);
            x[b] = s4;
          }
          if (more) load(kr, a.k, t + 8);
          // tokens behind the request's last one, and a second tile of another piece or of nobody
          const int held = min(own, i1 * BLK);
          if ((t + 2) * BLK > held) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if ((t + b) * BLK + 4 * g4 + i >= held) x[b][i] = -INFINITY;
          }
          float top = largest(x) * a.scale_log2;
          if (__builtin_amdgcn_ballot_w64(top > m + SLACK) != 0) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top), f = joined(m, m_new);
            m = m_new;
            l *= f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) O[dt] *= f;
          }
          bf16x8 ph, pl;
          float sum = 0.f;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][i], a.scale_log2, -m));
              sum += pv;
              __bf16 hi, lo;
              two_parts(pv, hi, lo);
              ph[4 * b + i] = hi;
              pl[4 * b + i] = lo;
            }
          l += sum;
          bf16x8 av[DT];
#pragma unroll
          for (int sp = 0; sp < NS; ++sp) {
            const uint4v w0 = piece(vr[0], sp), w1 = piece(vr[1], sp);
            av[2 * sp] = join(uint2v{w0[0], w0[1]}, uint2v{w1[0], w1[1]});
            av[2 * sp + 1] = join(uint2v{w0[2], w0[3]}, uint2v{w1[2], w1[3]});
          }
          if ((t + 2) * BLK > held) {                        // stale V may be a NaN pattern, which a weight of 0 does not remove
            uint4v keep;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const int tok = (t + (w >> 1)) * BLK + 4 * g4 + 2 * (w & 1);
              keep[w] = (tok < held ? 0x0000ffffu : 0u) | (tok + 1 < held ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) av[dt] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(uint4v, av[dt]) & keep);
          }
          if (more) load(vr, a.v, t + 8);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], ph, O[dt], 0, 0, 0);
            O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], pl, O[dt], 0, 0, 0);
          }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        // the four waves' states -> one
        __syncthreads();                                     // the stages (line A), or the states of the piece before, are done with
        float* st = (float*)stage_mem;
        if (g4 == 0) wave_ml[wv][col16] = make_float2(m, l);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(float4v*)(st + (wv * 16 + col16) * D + 16 * dt + 4 * g4) = O[dt];
        __syncthreads();
        const int64_t c = cut >= 0 ? shared_cut_b(a, cut) : shared_first(a, 1, r, g * G);
        for (int e = tid; e < G * D; e += SHARED_THREADS) {
          const int h = e / D, ch = e % D;
          float mm = LOWEST_REF, ll = 0.f, oo = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) mm = fmaxf(mm, wave_ml[w][h].x);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float2 ml = wave_ml[w][h];
            const float f = joined(ml.x, mm);
            ll += ml.y * f;
            oo += st[(w * 16 + h) * D + ch] * f;
          }
          a.part_o[(c + h) * 128 + ch] = oo;
          if (ch == 0) a.part_ml[c + h] = make_float2(mm, ll);
        }
      }
    }
  };

  if (turn * 2 < turns) {
    if (share_a >= 0) line_a();
    if (share_b >= 0) line_b();
  } else {
    if (share_b >= 0) line_b();
    if (share_a >= 0) line_a();
  }
}

// Joins the pieces of a request's two parts: a wave per (request, query head), two channels a lane.  Lane i looks up piece i (64 a
// round); the outputs of the first 16 are requested beside all references and sums, in one round trip.
template <int D>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedArgs a) {
  const int lane = threadIdx.x & 63;
  const int id = rfl(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (id >= a.n * a.Hq) return;
  const int r = id / a.Hq, hq = id - r * a.Hq, g = hq / a.G;
  const SharedRecord rec = a.rec[r];
  const bool lane_has = 2 * lane < D;
  const float* base = a.part_o + (lane_has ? 2 * lane : 0);
  const int h = hq - g * a.G, col = rec.a_col + h, cb = col / SHARED_COLS;
  const int n = rec.a_chunks + rec.b_chunks;
  float m = LOWEST_REF, l = 0.f;
  float2 o = {0.f, 0.f};
  for (int i0 = 0; i0 < n; i0 += 64) {
    // lane i: piece i0 + i, line A's first
    const int i = i0 + lane, here = min(64, n - i0);
    const bool on_a = i < rec.a_chunks, has = i < n;
    const int j = on_a ? i : i - rec.a_chunks;               // chunk
    const int64_t c = j == 0 ? shared_first(a, on_a ? 0 : 1, r, hq)
                      : on_a ? shared_cut_a(a, rec.a_extra + (g * (rec.a_chunks - 1) + j - 1) * rec.a_blocks + cb) + col - cb * SHARED_COLS
                             : shared_cut_b(a, rec.b_extra + g * (rec.b_chunks - 1) + j - 1) + h;
    const int c_lo = has ? (int)c : 0;                       // (columns of the workspace fit 32 bits)
    const float2 ml = has ? a.part_ml[c] : make_float2(LOWEST_REF, 0.f);
    constexpr int ROUND = 16;
    float2 x[ROUND];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < ROUND; ++k)
        x[k] = *(const float2*)(base + (int64_t)__builtin_amdgcn_readlane(c_lo, min(k0 + k, here - 1)) * 128);
    };
    load(0);                                                 // under way before the weights are known
    const float m_new = fmaxf(m, wave_max(ml.x)), f = joined(m, m_new), fx = has ? joined(ml.x, m_new) : 0.f;
    l = l * f + wave_sum(ml.y * fx);
    o.x *= f;
    o.y *= f;
    m = m_new;
    for (int k0 = 0;;) {
#pragma unroll
      for (int k = 0; k < ROUND; ++k) {
        const float w_k = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(fx), min(k0 + k, 63)));
        if (k0 + k < here && w_k != 0.f) {
          o.x = __builtin_fmaf(x[k].x, w_k, o.x);
          o.y = __builtin_fmaf(x[k].y, w_k, o.y);
        }
      }
      if ((k0 += ROUND) >= here) break;
      load(k0);
    }
  }
  if (lane_has) {
    const bool empty = n == 0;
    const float inv = a.out_scale / l;
    const int64_t at = (int64_t)id * D + 2 * lane;
    const float x = empty ? 0.f : o.x * inv, y = empty ? 0.f : o.y * inv;
    if (a.out_bf16) *(unsigned*)((unsigned short*)a.out + at) = (unsigned)float_to_bf16_bits(x) | ((unsigned)float_to_bf16_bits(y) << 16);
    else *(float2*)((float*)a.out + at) = make_float2(x, y);
  }
}

}  // namespace
