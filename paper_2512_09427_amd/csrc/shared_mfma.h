// Decode attention of a batch that shares prefixes, for gfx950.
//
// A request's softmax runs over its group's prefix and its own tokens.  Each of the two parts leaves a state of a query
// column (request, query head): reference m, sum l = sum 2^(s - m), O = sum 2^(s - m) V; states join by
//   M = max m_i,  out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i,
// so the prefix can be attended to by the queries of all its requests together: (requests x heads of a KV head's group)
// columns against its tokens, a dense contraction with reuse, where a request by itself only streams.
//
// Two lines of work.  Line A: items (prefix, KV head, block of SHARED_COLS columns), cut into chunks of pairs of 16-token tiles, a
// work-group's piece each.  Line B: items (request, KV head), each the pairs of tiles of the request's own tokens; the line is cut
// into shares, one for a wave, which streams it across the items in it, straight into registers.  Each piece of an item leaves
// its state in the workspace and shared_merge_kernel joins them.
//
// Both lines run at once, line A's matrix instructions beside line B's memory traffic: some work-groups take line A, the others line
// B.  Line B needs no more of them than fill the memory's rate (about 220 of 512), line A is as fast as it has work-groups; SHARED_TIMES
// says how long either takes and the plan divides them so that both end together.  The states of line A are as large as its
// columns (64 KiB a piece), so few long pieces are better than many short ones: with a piece for every work-group, 64 requests
// behind 4096 tokens wrote and read 25 MB of states beside 105 MB of K and V.  Line A is ordered (prefix, KV head, chunk, column
// block): the work-groups of an XCD read the same few chunks at a time, out of its L2.
#pragma once

#include <type_traits>

#include "kernels_common.h"
#include "prefixes.h"

namespace {

typedef const int64_t __attribute__((address_space(4))) const_i64s;

enum { SHARED_BF16_128, SHARED_FP8_128, SHARED_BF16_64 };
constexpr int SHARED_COLS = 128;          // columns of an item of line A: four waves of two 16-column tiles
constexpr int SHARED_CT = 2;
constexpr int SHARED_A_EXTRA = 5;         // start and end of a piece of line A, in pairs
// Pairs below which line A is not cut: at least 4, and SHARED_A_ROOT times the root of all its pairs.  A pair takes 0.7 us of a work-group that
// has its compute unit to itself, a piece 0.025 us of the memory's time for its states (128 columns, written and read), and
// 0.7 x + 0.025 U / x is least at 0.19 sqrt(U).  (8 at least: 8 requests behind 992 tokens 16.8 us, 14.6 with 4; 4 always: 16 behind
// 16 384 27.1 -> 31.9.)
constexpr float SHARED_A_LEAST = 4.f, SHARED_A_ROOT = 0.19f;
constexpr int SHARED_B_EXTRA = 2;         // start and end of an item of line B, in units
constexpr int SHARED_B_LEAST = 2;         // units that a wave is given at least, beside an item's start and end
// Microseconds: of a pair of line A for its work-group; of a pair of line B for its work-group while the memory has room (its
// bytes in flight over the latency), and for the whole chip at the memory's rate (16 KiB at 5.4 TB/s; 8 in the other formats).
struct SharedTimes {
  float a, b, b_least;
};
constexpr SharedTimes SHARED_TIMES[3] = {{1.3f, 0.65f, 0.003f}, {1.3f, 0.45f, 0.0015f}, {0.8f, 0.45f, 0.0015f}};
constexpr int SHARED_MAX_N = ODMA_SHARED_MAX_REQUESTS;
constexpr int SHARED_THREADS = 256, SHARED_WAVES = SHARED_THREADS / 64;

struct SharedRecord {                     // of a request, for the merge
  int32_t a_chunks, a_blocks, a_col;      // line A: chunks (0: it shares nothing) and column blocks of an item, its first column
  int32_t a_extra;                        // cut pieces (chunks behind the first) in front of its group's
  int32_t b_pos, b_units;                 // line B: place of its first head's item, units of an item
  int32_t pad0, pad1;
};
struct SharedShares {                     // how line B is dealt out (SharedLine): units, and waves of an XCD
  int32_t total, of_xcd;
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
  SharedShares* shares;
  float2* part_ml;                        // states of columns: reference and sum
  float* part_o;                          // [column][128]
};

// Columns of the workspace: first pieces of line A and of line B by (request, head); then line A's chunks behind the first, at most
// `workers` (SharedCut); then of every wave the piece of the item that its share begins inside of.
__device__ __forceinline__ int64_t shared_first(const SharedArgs& a, int line, int r, int hq) {
  return ((int64_t)line * a.n + r) * a.Hq + hq;
}
__device__ __forceinline__ int64_t shared_cut_a(const SharedArgs& a, int i) { return (int64_t)2 * a.n * a.Hq + (int64_t)i * a.cut_cols; }
__device__ __forceinline__ int64_t shared_cut_b(const SharedArgs& a, int w) {
  return (int64_t)2 * a.n * a.Hq + (int64_t)a.workers * a.cut_cols + (int64_t)w * a.G;
}

// a / b for 0 <= a, 0 < b and quotients below 2^20 (the reciprocal's error is less than one there)
__device__ __forceinline__ int small_quotient(int a, int b) {
  int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
  q -= q * b > a;
  q += (q + 1) * b <= a;
  return q;
}

// How line A with `units` pairs in `items` items is cut for `pieces` work-groups: into chunks of at most about `length`.  An item of T
// pairs has fewer than T / length chunks behind its first, all items together fewer than units / length, which is at
// most `pieces` (half of them where items abound, so that they are cut little).
struct SharedCut {
  float inv_length;
  int shift;                                                // costs count 2^shift pairs, so that the line's sum fits 30 bits
  __device__ __forceinline__ SharedCut(float units, int items, int pieces) {
    const float least = fmaxf(SHARED_A_LEAST, SHARED_A_ROOT * __builtin_amdgcn_sqrtf(units));
    const float length = fmaxf(units * 1.0005f * __builtin_amdgcn_rcpf((float)max(pieces - items, pieces / 2)), least);   // (the sum is within 2^-13)
    inv_length = __builtin_amdgcn_rcpf(length);
    shift = max((int)(__float_as_uint(units) >> 23) - 127 - 27, 0);
  }
  __device__ __forceinline__ int chunks(int T) const { return max((int)ceilf((float)T * inv_length), 1); }
};
// first unit of a chunk of an item of T units: chunks differ by one at most
__device__ __forceinline__ int chunk_start(int T, int chunks, int chunk) {
  const int base = T / chunks;
  return chunk * base + min(chunk, T - chunks * base);
}
// The N pieces of a group that begins at s on line A's cost and costs c are spread over it evenly: how many begin in front of x.
__device__ __forceinline__ int pieces_before(int x, int s, int c, int N) {
  return x <= s ? 0 : x >= s + c ? N : min((int)ceilf((float)(x - s) * (float)N / (float)c), N);   // (monotone in x)
}

// Line B: wave w's share is [start(w), start(w + 1)).  An item at s with T units has unit 0 at s and unit i at s + SHARED_B_EXTRA + i, and
// a unit belongs to the share that holds its position.
struct SharedLine {
  int total, waves;
  float inv;
  double step;
  __device__ __forceinline__ SharedLine(const SharedShares& s) : total(s.total), waves(8 * s.of_xcd) {
    step = (double)total / (double)waves;
    inv = (float)waves * __builtin_amdgcn_rcpf((float)total);
  }
  __device__ __forceinline__ int start(int w) const { return w >= waves ? total : (int)((double)w * step); }
  __device__ __forceinline__ int holder(int pos) const {
    int w = min((int)((float)pos * inv), waves - 1);
    while (start(w) > pos) --w;                              // (the estimate is within a few)
    while (start(w + 1) <= pos) ++w;
    return w;
  }
};
__device__ __forceinline__ int units_before(int x, int s, int T) {
  return x <= s ? 0 : min(max(x - s - SHARED_B_EXTRA, 1), T);
}

template <bool HIGH_HALF>
__device__ __forceinline__ unsigned widen_e4m3x2(unsigned w) {
  typedef float float2v __attribute__((ext_vector_type(2)));
  const float2v f = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HIGH_HALF);
  return (__float_as_uint(f[0]) >> 16) | (__float_as_uint(f[1]) & 0xffff0000u);
}

struct SharedPlan {
  // requests
  int32_t own[SHARED_MAX_N];              // tokens that it reads itself; SHARES: and all of its group's shared ones with the group
  int32_t base[SHARED_MAX_N];             // block of the first of them, or its place in the request's row of the block table
  int32_t b_pos[SHARED_MAX_N + 1];        // units of line B in front of it
  // groups
  int32_t start[SHARED_MAX_N + 1];        // first request
  int32_t tiles[SHARED_MAX_N];            // of the shared part
  int32_t first_block[SHARED_MAX_N];      // (contiguous)
  int32_t reader[SHARED_MAX_N];           // its first request that holds all of the shared part
  int32_t a_pos[SHARED_MAX_N + 1];        // cost of line A in front of it, or pieces where every work-group gets one
  int32_t a_extra[SHARED_MAX_N];          // cut pieces in front of it
  float units[SHARED_WAVES][2];
  int32_t items[SHARED_WAVES], sums[SHARED_WAVES][4];
};
constexpr int SHARES = (int)0x80000000;

__device__ __forceinline__ int tiles_of(int tokens) { return (int)(((int64_t)tokens + BLK - 1) / BLK); }
__device__ __forceinline__ int column_blocks(int count, int G) { return (count * G + SHARED_COLS - 1) / SHARED_COLS; }

// A score in exponent units, rounded: a product that went into the subtraction of the reference unrounded would differ from the
// reference (the largest of these numbers) by its rounding, which is more than an exponent holds where scores are large.
__device__ __forceinline__ float in_exponent_units(float score, float scale_log2) {
#pragma clang fp contract(off)
  return score * scale_log2;
}

// Factor of a state joined to another.  At least the smallest number: 0 would make an infinite sum NaN.
__device__ __forceinline__ float joined(float m, float m_new) { return fmaxf(__builtin_amdgcn_exp2f(m - m_new), 0x1p-149f); }

// A weight as N bf16 parts: all but the last cut off, the last rounded (off by 2^-8 of it at most for N = 1, 2^-16 for 2, exact for 3, but
// for a least part of 2^-126).  None is negative, nor 0 unless the weight is (a weight of less than 2^-126 is): an infinite V times the
// parts is that infinity, as times the weight.  Beside the weights' sum, at least 1 in the end, the least parts are nothing.
template <int N>
__device__ __forceinline__ void weight_parts(float w, bf16x8 (&parts)[N], int at) {
  float rest = w;
#pragma unroll
  for (int k = 0; k < N - 1; ++k) {
    const unsigned bits = __float_as_uint(rest) & 0xffff0000u;
    parts[k][at] = __builtin_bit_cast(__bf16, (unsigned short)(bits >> 16));
    rest = fmaxf(rest - __uint_as_float(bits), fminf(w, 0x1p-126f));
  }
  parts[N - 1][at] = (__bf16)rest;
}

// inclusive sums over the lanes of a wave, by moves inside rows of 16 and broadcasts between them
template <typename T>
__device__ __forceinline__ T lanes_sum(T x) {
  auto moved = [](T v, auto ctrl, auto rows) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  using std::integral_constant;
  x += moved(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
  x += moved(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return x;
}

// the largest over the lanes of a wave
__device__ __forceinline__ float lanes_max(float x) {
  auto moved = [](float v, auto ctrl, auto rows) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  using std::integral_constant;
  x = fmaxf(x, moved(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{}));
  x = fmaxf(x, moved(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{}));
  x = fmaxf(x, moved(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{}));
  x = fmaxf(x, moved(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{}));
  x = fmaxf(x, moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}));
  x = fmaxf(x, moved(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Last entry of pos[0 .. n) (which does not decrease, and begins with 0) that is at most x >= 0; n <= 4096.
__device__ __forceinline__ int last_at_most(const int32_t* pos, int n, int x) {
  const int lane = threadIdx.x & 63;
  auto probe = [&](int i) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < n && pos[min(i, n - 1)] <= x)); };
  int lo = 0;
  if (n > 64) {
    const int span = (n + 63) / 64;
    lo = (probe(lane * span) - 1) * span;
    const int last = min(span, n - lo);
    return lo + __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < last && pos[min(lo + lane, n - 1)] <= x)) - 1;
  }
  return probe(lane) - 1;
}

// EXACT: the weights go through the matrix cores as three bf16 parts, all their bits; for fp32 results.  Otherwise as one part in
// line A (half a bf16 step of one term of the sum, as the rounding of a bf16 result is of the whole) and as two in line B, where
// matrix instructions wait for memory in any case.  Two parts in line A as well would bring bf16 results from 2.2e-3 to the 1.7e-3 that their
// own rounding is, and cost 14.5 -> 15.3 us for 8 requests behind 1000 tokens, 32.0 -> 34.3 for 64 behind 4096, 95.4 -> 125.8 for 256
// behind 16 384 and 31.0 -> 32.6 for 128 with fp8 pages.
template <int FMT, bool PAGED, bool EXACT>
__global__ __launch_bounds__(SHARED_THREADS, 2) void shared_parts_kernel(SharedArgs a) {
  constexpr bool FP8 = FMT == SHARED_FP8_128;
  constexpr int D = FMT == SHARED_BF16_64 ? 64 : 128;
  constexpr int NS = D / 32, DT = D / 16;                   // 32-channel steps, 16-channel groups
  constexpr int TILE_BYTES = BLK * D * (FP8 ? 1 : 2), LOADS = TILE_BYTES / 1024;
  constexpr int K_STAGE = 2 * NS * 1024, STAGE_BYTES = 2 * K_STAGE;
  constexpr int CT = SHARED_CT;
  constexpr int PARTS_A = EXACT ? 3 : 1, PARTS_B = EXACT ? 3 : 2;
  constexpr int V_AHEAD = D == 64 ? DT : EXACT ? 0 : 5;       // V operands that there are registers for in front of their weights
  constexpr float SLACK = 8.0f;                             // exponent units by which a score may exceed the reference
  __shared__ __attribute__((aligned(16))) char stage_mem[2 * STAGE_BYTES];
  __shared__ SharedPlan plan;
  const int tid = threadIdx.x, lane = tid & 63, wv = rfl(tid >> 6);
  const int col16 = lane & 15, g4 = lane >> 4;
  const unsigned lane16 = lane * 16;
  const int G = a.G;

  // ---- plan: every work-group for itself (a launch of its own would be one work-group's round trips on an empty chip).  One
  // round of loads, then LDS alone.
  const int per = (a.n + SHARED_THREADS - 1) / SHARED_THREADS, perp = (a.n_prefixes + SHARED_THREADS - 1) / SHARED_THREADS;
  const int r0 = min(tid * per, a.n), r1 = min(r0 + per, a.n);
  const int p0 = min(tid * perp, a.n_prefixes), p1 = min(p0 + perp, a.n_prefixes);
  for (int r = tid; r < a.n; r += SHARED_THREADS) {
    plan.own[r] = max(a.lengths[r], 0);
    if (!PAGED) plan.base[r] = (int)(a.offsets[r] / BLK);
  }
  for (int p = tid; p <= a.n_prefixes; p += SHARED_THREADS) {
    plan.start[p] = min(max(a.prefix_start[p], 0), a.n);
    if (p < a.n_prefixes) {
      plan.tiles[p] = shared_tokens(a.prefix_lengths[p]) / BLK;
      if (!PAGED) plan.first_block[p] = (int)(a.prefix_offsets[p] / BLK);
      plan.reader[p] = a.n;
    }
  }
  __syncthreads();
  auto group_blocks = [&](int p) { return plan.tiles[p] ? column_blocks(max(plan.start[p + 1] - plan.start[p], 0), G) : 0; };
  float units[2] = {0.f, 0.f};                               // pairs of lines A and B, per KV head
  int items = 0;                                             // of line A
  for (int r = r0; r < r1; ++r) {
    const int len = plan.own[r], p = prefix_of(plan.start, a.n_prefixes, r), shared = p >= 0 ? plan.tiles[p] * BLK : 0;
    const bool shares = shared > 0 && len >= shared;
    const int own = shares ? len - shared : len;
    plan.own[r] = own | (shares ? SHARES : 0);
    if (shares) atomicMin(&plan.reader[p], r);
    // its own slab, behind its shared blocks in a row of the table; a request shorter than the shared part reads its group's prefix
    if (PAGED) plan.base[r] = shares ? shared / BLK : 0;
    else if (shared > 0 && !shares) plan.base[r] = plan.first_block[p];
    units[1] += (float)(tiles_of(own) / 2 + 1);
  }
  for (int p = p0; p < p1; ++p) {
    const int blocks = group_blocks(p);
    units[0] += (float)blocks * (float)((plan.tiles[p] + 1) / 2);
    items += blocks;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) units[i] = lanes_sum(units[i]);
  items = lanes_sum(items);
  if (lane == 63) {
#pragma unroll
    for (int i = 0; i < 2; ++i) plan.units[wv][i] = units[i];
    plan.items[wv] = items;
  }
  __syncthreads();
  units[0] = units[1] = 0.f;
  items = 0;
#pragma unroll
  for (int w = 0; w < SHARED_WAVES; ++w) {
#pragma unroll
    for (int i = 0; i < 2; ++i) units[i] += plan.units[w][i];
    items += plan.items[w];
  }
  units[0] *= (float)a.Hkv;
  units[1] *= (float)a.Hkv;
  // work-groups for line A: as many as end with line B
  const SharedTimes times = SHARED_TIMES[FMT];
  const float time_a = (units[0] + (float)(items * a.Hkv * SHARED_A_EXTRA)) * times.a, time = fmaxf((time_a + units[1] * times.b) * __builtin_amdgcn_rcpf((float)a.workers), units[1] * times.b_least);
  const int for_a = rfl(min(max((int)(time_a * __builtin_amdgcn_rcpf(fmaxf(time, 1e-3f)) + 7.f) / 8 * 8, 8), a.workers));
  const SharedCut cut_a(units[0], items * a.Hkv, for_a);
  // A unit of line B: 2^shift_b pairs, so that the line fits 30 bits (it always does unless tables name the same blocks over and over).
  const int shift_b = rfl(max((int)(__float_as_uint(units[1]) >> 23) - 127 - 28, 0));
  auto pairs_b = [&](int r) { return (tiles_of(plan.own[r] & ~SHARES) + 1) / 2; };
  auto units_b = [&](int r) { return (pairs_b(r) + (1 << shift_b) - 1) >> shift_b; };
  int sum[4] = {0, 0, 0, 0};
  struct Entry {
    int cost, extra, pieces;
  };
  auto group_entry = [&](int p) {
    const int blocks = group_blocks(p), pairs = (plan.tiles[p] + 1) / 2, chunks = cut_a.chunks(pairs);
    if (!blocks) return Entry{0, 0, 0};
    return Entry{(int)((int64_t)a.Hkv * blocks * (pairs + chunks * SHARED_A_EXTRA) >> cut_a.shift) + 1, a.Hkv * blocks * (chunks - 1), a.Hkv * blocks * chunks};
  };
  auto request_cost = [&](int r) {
    const int T = units_b(r);
    return T ? a.Hkv * (T + SHARED_B_EXTRA) : 0;
  };
  for (int p = p0; p < p1; ++p) {
    const Entry e = group_entry(p);
    sum[0] += e.cost;
    sum[1] += e.extra;
    sum[3] += e.pieces;
  }
  for (int r = r0; r < r1; ++r) sum[2] += request_cost(r);
  int before[4], total[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) before[i] = lanes_sum(sum[i]);
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < 4; ++i) plan.sums[wv][i] = before[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    before[i] -= sum[i];
    total[i] = 0;
#pragma unroll
    for (int w = 0; w < SHARED_WAVES; ++w) {
      const int x = plan.sums[w][i];
      if (w < wv) before[i] += x;
      total[i] += x;
    }
    total[i] = rfl(total[i]);
  }
  // As a rule there are no more pieces than work-groups for them: one each, whatever they cost.
  const bool one_each = total[3] <= for_a;
  const int total_a = one_each ? total[3] : total[0];
  for (int p = p0; p < p1; ++p) {
    const Entry e = group_entry(p);
    plan.a_pos[p] = one_each ? before[3] : before[0];
    plan.a_extra[p] = before[1];
    before[0] += e.cost;
    before[1] += e.extra;
    before[3] += e.pieces;
  }
  for (int r = r0; r < r1; ++r) {
    plan.b_pos[r] = before[2];
    before[2] += request_cost(r);
  }
  if (tid == 0) {
    plan.a_pos[a.n_prefixes] = total_a;
    plan.b_pos[a.n] = total[2];
  }
  __syncthreads();
  // Shares.  XCD x (work-groups x, x + 8, ..) has neighbouring ones, which read the same heads.  Line A goes to the first work-groups of
  // every XCD, line B to the last, as many as have work.
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, turns = a.workers >> 3;
  const int used_a = rfl(min(total[3], for_a)), ja = (used_a + 7) >> 3;
  const int jb = rfl(total[2] ? min(total[2] / (8 * SHARED_WAVES * (SHARED_B_LEAST + SHARED_B_EXTRA)) + 1, turns) : 0);
  // Line B leaves the work-groups of line A alone, unless they are all there are.
  const SharedShares shares = {total[2], SHARED_WAVES * min(jb, ja < turns ? turns - ja : turns)};
  const int share_a = turn < ja && xcd * ja + turn < used_a ? xcd * ja + turn : -1;
  const int in_xcd_b = SHARED_WAVES * (turns - 1 - turn) + wv;   // line B: the wave's number on its XCD
  if (blockIdx.x == gridDim.x - 1) {                        // for the merge
    for (int r = tid; r < a.n; r += SHARED_THREADS) {
      SharedRecord rec = {0, 0, 0, 0, plan.b_pos[r], units_b(r), 0, 0};
      if (plan.own[r] & SHARES) {
        const int p = prefix_of(plan.start, a.n_prefixes, r);
        rec.a_chunks = cut_a.chunks((plan.tiles[p] + 1) / 2);
        rec.a_blocks = group_blocks(p);
        rec.a_col = (r - plan.start[p]) * G;
        rec.a_extra = plan.a_extra[p];
      }
      a.rec[r] = rec;
    }
    if (tid == 0) *a.shares = shares;
  }

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

  // ================= line A
  auto line_a = [&]() {
    bf16x8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;
    const double step_a = (double)total_a / (double)used_a;
    const int x0 = rfl((int)((double)share_a * step_a)), x1 = rfl(share_a + 1 >= used_a ? total_a : (int)((double)(share_a + 1) * step_a));
    for (int p = rfl(last_at_most(plan.a_pos, a.n_prefixes, x0)); p < a.n_prefixes; ++p) {
      const int pos = rfl(plan.a_pos[p]), cost = rfl(plan.a_pos[p + 1]) - pos, reader = rfl(plan.reader[p]);
      if (pos >= x1) break;
      if (!cost || reader == a.n) continue;                  // (nobody attends to it)
      const int begin = rfl(plan.start[p]), count = rfl(plan.start[p + 1]) - begin;
      const int n_tiles = rfl(plan.tiles[p]), pairs = (n_tiles + 1) / 2, chunks = rfl(cut_a.chunks(pairs));
      const int blocks = rfl(column_blocks(count, G)), per_head = chunks * blocks, n_pieces = a.Hkv * per_head, n_cols = count * G;
      const int64_t base_block = PAGED ? 0 : rfl(plan.first_block[p]);
      const const_i32* bt_row = as_constant(PAGED ? a.bt + (int64_t)reader * a.bt_stride : nullptr);
      const int last = rfl(pieces_before(x1, pos, cost, n_pieces));
      for (int id = rfl(pieces_before(x0, pos, cost, n_pieces)); id < last; ++id) {
        const int g = rfl(small_quotient(id, per_head)), chunk = rfl(small_quotient(id - g * per_head, blocks));
        const int cb = id - g * per_head - chunk * blocks;
        const int i0 = rfl(chunk_start(pairs, chunks, chunk)), i1 = rfl(chunk_start(pairs, chunks, chunk + 1));
        const int cut = chunk ? rfl(plan.a_extra[p]) + (g * (chunks - 1) + chunk - 1) * blocks + cb : -1;
        const int c0 = cb * SHARED_COLS + wv * 16 * CT;
        const bool active = rfl(c0 < n_cols);
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
        // A column's reference m is subtracted behind the products: in the accumulators of the scores, one that lies far below the next
        // pair's scores would leave them no bits.  The sum of its weights is one more row of P V, with V = 1.
        float m[CT];
        float4v l[CT], O[CT][DT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          m[ct] = LOWEST_REF;
          l[ct] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) O[ct][dt] = float4v{0.f, 0.f, 0.f, 0.f};
        }

        // loading: waves 0 and 1 bring K of the first and second tile of a pair, 2 and 3 V.  A second tile that does not exist
        // re-reads the first with its V zeroed (its scores are masked).  K runs a pair ahead of V: load j is pair i0 + j of K and
        // i0 + j - 1 of V.
        const bool loads_v = wv >= 2;
        const int which = wv & 1, behind = loads_v ? 1 : 0;
        const char* src_base = (loads_v ? a.v : a.k) + plane;
        auto pair_of = [&](int j) { return min(max(i0 + j - behind, i0), i1 - 1); };
        auto tile_of = [&](int j) { return min(2 * pair_of(j) + which, n_tiles - 1); };
        int blk_next = 0;
        auto lookup = [&](int j) {
          if (PAGED) blk_next = bt_row[tile_of(j)];
        };
        auto issue = [&](uint4v (&rg)[LOADS], int j) {
          const char* src = src_base + (PAGED ? (int64_t)blk_next : base_block + tile_of(j)) * TILE_BYTES;
#pragma unroll
          for (int i = 0; i < LOADS; ++i) rg[i] = *(const uint4v*)(src + i * 1024 + lane16);
        };
        auto write_stage = [&](const uint4v (&rg)[LOADS], int j) {
          char* st = stage_mem + ((j - behind) & 1) * STAGE_BYTES;
          if (!loads_v) {
#pragma unroll
            for (int sp = 0; sp < NS; ++sp) *(uint4v*)(st + which * NS * 1024 + sp * 1024 + lane16) = piece(rg, sp);
          } else {
            char* dst = st + K_STAGE + lane16 + which * 8;
            const bool absent = 2 * pair_of(j) + which >= n_tiles;
#pragma unroll
            for (int sp = 0; sp < NS; ++sp) {
              const uint4v w = piece(rg, sp);
              *(uint2v*)(dst + (2 * sp) * 1024) = uint2v{w[0], w[1]};
              *(uint2v*)(dst + (2 * sp + 1) * 1024) = uint2v{w[2], w[3]};
            }
            if (__builtin_expect(absent, 0))
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) *(uint2v*)(dst + dt * 1024) = uint2v{0u, 0u};
          }
        };
        auto read_k = [&](bf16x8 (&kk)[NS], int j, int b) {   // tile b of pair i0 + j
          const char* st = stage_mem + (j & 1) * STAGE_BYTES + lane16;
#pragma unroll
          for (int sp = 0; sp < NS; ++sp) kk[sp] = *(const bf16x8*)(st + b * NS * 1024 + sp * 1024);
        };
        auto scores = [&](float4v (&x)[CT][2], const bf16x8 (&kk)[NS], int b) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            float4v s4 = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int sp = 0; sp < NS; ++sp) s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[sp], qreg[ct][sp], s4, 0, 0, 0);
            x[ct][b] = s4;
          }
        };
        auto settle = [&](float4v (&x)[CT][2], int pr) {      // scores of pair pr: masked, and above the references by SLACK at most
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) x[ct][b][i] = in_exponent_units(x[ct][b][i], a.scale_log2);
          if (2 * pr + 1 >= n_tiles) {
            asm volatile("");                                // (a branch: once an item, against eight selects a pair)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) x[ct][1] = float4v{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          }
          // (Each tile by itself: a lane's columns are of different requests, and a NaN of one must not hide the other's rise.)
          float top[CT];
          bool above = false;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            top[ct] = largest(x[ct]);
            above |= top[ct] > m[ct] + SLACK;
          }
          if (__builtin_amdgcn_ballot_w64(above) != 0) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
              float up = fmaxf(top[ct], __shfl_xor(top[ct], 16));
              up = fmaxf(up, __shfl_xor(up, 32));
              // (A column moves for its own scores alone: its bits do not depend on its neighbours', which may be an empty place's.)
              const float m_new = up > m[ct] + SLACK ? up : m[ct], f = m_new > m[ct] ? joined(m[ct], m_new) : 1.f;
              m[ct] = m_new;
              l[ct] *= f;
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) O[ct][dt] *= f;
            }
          }
        };
        // Pair pr: its weights (vector instructions) beside the scores of the pair behind it (matrix instructions), then P V.
        auto compute = [&](float4v (&x)[CT][2], float4v (&ahead)[CT][2], int pr) {
          // LDS first: K of the pair behind this one and V of this one are on their way while the references are looked at
          bf16x8 k0[NS], k1[NS], av[DT];
          const char* st = stage_mem + ((pr - i0) & 1) * STAGE_BYTES + K_STAGE + lane16;
          read_k(k0, pr + 1 - i0, 0);
#pragma unroll
          for (int dt = 0; dt < V_AHEAD; ++dt) av[dt] = *(const bf16x8*)(st + dt * 1024);
          __builtin_amdgcn_sched_barrier(0);
          settle(x, pr);
          read_k(k1, pr + 1 - i0, 1);
          scores(ahead, k0, 0);
          scores(ahead, k1, 1);
          bf16x8 w[CT][PARTS_A];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) weight_parts(__builtin_amdgcn_exp2f(x[ct][b][i] - m[ct]), w[ct], 4 * b + i);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int k = 0; k < PARTS_A; ++k) l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w[ct][k], l[ct], 0, 0, 0);
#pragma unroll
          for (int dt = V_AHEAD; dt < DT; ++dt) av[dt] = *(const bf16x8*)(st + dt * 1024);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
              for (int k = 0; k < PARTS_A; ++k) O[ct][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], w[ct][k], O[ct][dt], 0, 0, 0);
        };
        // pipeline: load j + 3 is under way while pair j is computed; load j + 2 goes from registers into its stage behind it, where
        // pair j + 1 finds it, and one barrier per pair makes it visible
        uint4v ra[LOADS], rb[LOADS];
        float4v xa[CT][2], xb[CT][2];
        lookup(0);
        issue(ra, 0);
        lookup(1);
        issue(rb, 1);
        lookup(2);
        __syncthreads();                                     // the stages of the piece before are done with
        write_stage(ra, 0);
        issue(ra, 2);
        lookup(3);
        __syncthreads();
        if (active) {
          bf16x8 kk[NS];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            read_k(kk, 0, b);
            scores(xa, kk, b);
          }
        }
        write_stage(rb, 1);
        __syncthreads();
        auto step = [&](uint4v (&near)[LOADS], uint4v (&far)[LOADS], float4v (&x)[CT][2], float4v (&ahead)[CT][2], int pr) {
          issue(far, pr - i0 + 3);
          lookup(pr - i0 + 4);
          if (active) compute(x, ahead, pr);
          write_stage(near, pr - i0 + 2);
          __syncthreads();
        };
        for (int pr = i0;;) {
          step(ra, rb, xa, xb, pr);
          if (++pr == i1) break;
          step(rb, ra, xb, xa, pr);
          if (++pr == i1) break;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if (!ok[ct]) continue;
          const int64_t c = cut >= 0 ? shared_cut_a(a, cut) + wv * 16 * CT + 16 * ct + col16 : shared_first(a, 0, row[ct], head[ct]);
          if (g4 == 0) a.part_ml[c] = make_float2(m[ct], l[ct][0]);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) *(float4v*)(a.part_o + c * 128 + 16 * dt + 4 * g4) = O[ct][dt];
        }
      }
    }
  };

  // ================= line B: every wave streams its share
  auto line_b = [&]() {
    const SharedLine line(shares);
    if (in_xcd_b >= shares.of_xcd) return;
    const int w = xcd * shares.of_xcd + in_xcd_b;
    const int x0 = rfl(line.start(w)), x1 = rfl(line.start(w + 1));
    struct Item {
      int r, g, i0, i1;                                     // pairs [i0, i1) of the request's own tokens
      int own, base;
    };
    // the first item at or behind (r, g) that has pairs in the share; r = n: there is none
    auto item_from = [&](int r, int g) {
      Item it = {a.n, 0, 0, 0, 0, 0};
      for (; r < a.n; ++r, g = 0) {
        const int pos = rfl(plan.b_pos[r]), T = rfl(units_b(r));
        if (pos >= x1) break;
        if (rfl(plan.b_pos[r + 1]) <= x0 || T == 0) continue;
        for (; g < a.Hkv; ++g) {
          const int s = pos + g * (T + SHARED_B_EXTRA), u0 = units_before(x0, s, T), u1 = units_before(x1, s, T);
          if (u0 < u1) {
            it = Item{r, g, u0 << shift_b, min(u1 << shift_b, rfl(pairs_b(r))), rfl(plan.own[r]) & ~SHARES, rfl(plan.base[r])};
            return it;
          }
          if (s >= x1) return it;
        }
      }
      return it;
    };
    const int first = rfl(last_at_most(plan.b_pos, a.n, x0));
    const int first_pos = rfl(plan.b_pos[first]), first_T = rfl(units_b(first));
    Item cur = item_from(first, first_T ? rfl(small_quotient(x0 - first_pos, first_T + SHARED_B_EXTRA)) : 0);
    if (cur.r >= a.n) return;
    auto load_q = [&](bf16x8 (&q)[NS], const Item& it) {
      const unsigned short* qp = a.q + ((int64_t)it.r * a.Hq + it.g * G + min(col16, G - 1)) * D + 8 * g4;
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
        q[st] = col16 < G ? *(const bf16x8*)(qp + 32 * st) : z;
      }
    };
    // the tiles of pair pr (the first one again where there is no second)
    auto blocks_of = [&](int64_t (&at)[2], const Item& it, int pr) {
      const int tiles = tiles_of(it.own);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int t = min(2 * pr + b, tiles - 1);
        at[b] = (int64_t)it.g * a.head_stride + (PAGED ? (int64_t)as_constant(a.bt + (int64_t)it.r * a.bt_stride)[it.base + t] : (int64_t)it.base + t) * TILE_BYTES;
      }
    };
    uint4v kr[2][LOADS], vr[2][LOADS];
    auto load = [&](uint4v (&to)[2][LOADS], const char* pool, const int64_t (&at)[2]) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) to[b][i] = __builtin_nontemporal_load((const uint4v*)(pool + at[b] + lane16 + i * 1024));
    };
    bf16x8 qreg[NS], qnext[NS];
    int64_t at[2];
    load_q(qnext, cur);
    blocks_of(at, cur, cur.i0);
    load(kr, a.k, at);
    load(vr, a.v, at);
    while (cur.r < a.n) {
      const Item next = cur.g + 1 < a.Hkv ? item_from(cur.r, cur.g + 1) : item_from(cur.r + 1, 0);
#pragma unroll
      for (int st = 0; st < NS; ++st) qreg[st] = qnext[st];
      if (next.r < a.n) load_q(qnext, next);
      float m = LOWEST_REF, l = 0.f;
      float4v O[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[dt] = float4v{0.f, 0.f, 0.f, 0.f};
      for (int pr = cur.i0; pr < cur.i1; ++pr) {
        // the loads of the pair behind this one, of this item or the next, go out as soon as their registers are free
        const bool inside = pr + 1 < cur.i1, more = inside || next.r < a.n;
        if (inside) blocks_of(at, cur, pr + 1);
        else if (more) blocks_of(at, next, next.i0);
        float4v x[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float4v s4 = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int sp = 0; sp < NS; ++sp)
            s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, piece(kr[b], sp)), qreg[sp], s4, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[b][i] = in_exponent_units(s4[i], a.scale_log2);
        }
        if (more) load(kr, a.k, at);
        const int t0 = 2 * pr * BLK;
        const bool ragged = t0 + 2 * BLK > cur.own;           // some tokens of the pair are not there
        if (ragged) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (t0 + b * BLK + 4 * g4 + i >= cur.own) x[b][i] = -INFINITY;
        }
        float top = largest(x);
        if (__builtin_amdgcn_ballot_w64(top > m + SLACK) != 0) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float m_new = fmaxf(m, top), f = joined(m, m_new);
          m = m_new;
          l *= f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) O[dt] *= f;
        }
        bf16x8 w_parts[PARTS_B];
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float pv = __builtin_amdgcn_exp2f(x[b][i] - m);
            sum += pv;
            weight_parts(pv, w_parts, 4 * b + i);
          }
        l += sum;
        bf16x8 av[DT];
#pragma unroll
        for (int sp = 0; sp < NS; ++sp) {
          const uint4v w0 = piece(vr[0], sp), w1 = piece(vr[1], sp);
          av[2 * sp] = join(uint2v{w0[0], w0[1]}, uint2v{w1[0], w1[1]});
          av[2 * sp + 1] = join(uint2v{w0[2], w0[3]}, uint2v{w1[2], w1[3]});
        }
        if (ragged) {                                          // stale V may be a NaN pattern, which a weight of 0 does not remove
          uint4v keep;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tok = t0 + (i >> 1) * BLK + 4 * g4 + 2 * (i & 1);
            keep[i] = (tok < cur.own ? 0x0000ffffu : 0u) | (tok + 1 < cur.own ? 0xffff0000u : 0u);
          }
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) av[dt] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(uint4v, av[dt]) & keep);
        }
        if (more) load(vr, a.v, at);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int k = 0; k < PARTS_B; ++k) O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[dt], w_parts[k], O[dt], 0, 0, 0);
      }
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (col16 < G) {
        const int64_t c = (cur.i0 ? shared_cut_b(a, w) : shared_first(a, 1, cur.r, cur.g * G)) + col16;
        if (g4 == 0) a.part_ml[c] = make_float2(m, l);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(float4v*)(a.part_o + c * 128 + 16 * dt + 4 * g4) = O[dt];
      }
      cur = next;
    }
  };

  if (share_a >= 0) line_a();
  line_b();
}

// Joins the pieces of a request's two parts: a wave per (request, HEADS query heads of a KV head), two channels a lane.  Lane i looks up
// piece i (64 a round); the outputs of the first ROUND are requested beside all references and sums, in one round trip.  Bound
// by its chain of round trips (record, states) and, where there are many, by the states' bytes.  A head's columns lie behind one another
// in all pieces (a column block that is not the last is whole).
// Where a prefix is long beside few heads, WAVES = 4 waves of a work-group take a quarter of the pieces each.
template <int D, int HEADS, int WAVES>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedArgs a) {
  static_assert(HEADS == 1 || WAVES == 1, "a wave per head hands its state on");
  __shared__ float4 handed[WAVES][64];                       // reference, sum, two channels of each lane
  constexpr int ROUND = HEADS == 1 ? 8 : 4;                  // (16: 256 requests behind 500 tokens 52.2 -> 54.4 us, 4: 16 behind 16 384 25.6 -> 28.0)
  const int lane = threadIdx.x & 63;
  const int wave = rfl(threadIdx.x >> 6), id = WAVES > 1 ? (int)blockIdx.x : rfl(blockIdx.x * 4 + wave), parts = (a.G + HEADS - 1) / HEADS;   // waves of a KV head
  const int rg = rfl(small_quotient(id, parts)), r = rfl(small_quotient(rg, a.Hkv)), g = rg - r * a.Hkv, h0 = (id - rg * parts) * HEADS;
  if (r >= a.n) return;
  const SharedRecord rec = a.rec[r];
  const SharedLine line(*a.shares);
  const int heads = min(HEADS, a.G - h0);
  // line B: the waves from the one that holds its first unit to the one that holds its last
  const int s = rec.b_pos + g * (rec.b_units + SHARED_B_EXTRA), w0 = rec.b_units ? rfl(line.holder(s)) : 0;
  const int n_b = rec.b_units ? rfl(line.holder(s + (rec.b_units > 1 ? SHARED_B_EXTRA + rec.b_units - 1 : 0))) - w0 + 1 : 0;
  const int n = rfl(rec.a_chunks + n_b);
  const int share = WAVES > 1 ? (n + WAVES - 1) / WAVES : n, begin = WAVES > 1 ? min(wave * share, n) : 0, end = min(begin + share, n);
  const int a_stride = rec.a_blocks * a.cut_cols, a_cut = (int)shared_cut_a(a, rec.a_extra + g * (rec.a_chunks - 1) * rec.a_blocks) + rec.a_col + h0;
  const bool lane_has = 2 * lane < D;
  const unsigned lane_at = lane_has ? lane * 8u : 0u;        // (columns of the workspace fit 23 bits, their bytes 32)
  float m[HEADS], l[HEADS];
  float2 o[HEADS];
#pragma unroll
  for (int h = 0; h < HEADS; ++h) {
    m[h] = LOWEST_REF;
    l[h] = 0.f;
    o[h] = make_float2(0.f, 0.f);
  }
  for (int i0 = begin; i0 < end; i0 += 64) {
    // lane i: piece i0 + i, line A's first
    const int i = i0 + lane, here = min(64, end - i0);
    const bool on_a = i < rec.a_chunks;
    const int j = on_a ? i : i - rec.a_chunks, w = w0 + j;    // chunk; or wave, by its distance from the first
    int c = j == 0 ? (int)shared_first(a, on_a ? 0 : 1, r, g * a.G + h0) : on_a ? a_cut + (j - 1) * a_stride : (int)shared_cut_b(a, w) + h0;
    // (a share shorter than an item's start may hold none of its units)
    const bool has = i < end && (on_a || j == 0 || units_before(line.start(w), s, rec.b_units) < units_before(line.start(w + 1), s, rec.b_units));
    if (!has) c = 0;
    float2 ml[HEADS], x[HEADS][ROUND];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) ml[h] = has ? a.part_ml[c + min(h, heads - 1)] : make_float2(LOWEST_REF, 0.f);
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < ROUND; ++k) {
        const unsigned at = (unsigned)__builtin_amdgcn_readlane(c, min(k0 + k, here - 1)) * 512u + lane_at;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) x[h][k] = *(const float2*)((const char*)a.part_o + at + (h < heads ? h * 512u : 0u));
      }
    };
    load(0);                                                 // under way before the weights are known
    float fx[HEADS];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      const float m_new = fmaxf(m[h], lanes_max(ml[h].x)), f = joined(m[h], m_new);
      fx[h] = has ? joined(ml[h].x, m_new) : 0.f;
      l[h] = l[h] * f + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(lanes_sum(ml[h].y * fx[h])), 63));
      o[h].x *= f;
      o[h].y *= f;
      m[h] = m_new;
    }
    for (int k0 = 0;;) {
#pragma unroll
      for (int k = 0; k < ROUND; ++k)
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
          const float w_k = k0 + k < here ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(fx[h]), min(k0 + k, 63))) : 0.f;
          const bool there = w_k != 0.f;                     // (a weight is 2^-149 at least; what is not there may hold anything)
          o[h].x = __builtin_fmaf(there ? x[h][k].x : 0.f, w_k, o[h].x);
          o[h].y = __builtin_fmaf(there ? x[h][k].y : 0.f, w_k, o[h].y);
        }
      if ((k0 += ROUND) >= here) break;
      load(k0);
    }
  }
  if (WAVES > 1) {
    if (wave) handed[wave][lane] = make_float4(m[0], l[0], o[0].x, o[0].y);
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      const float4 x = handed[w][lane];
      const float m_new = fmaxf(m[0], x.x), f = joined(m[0], m_new), g = joined(x.x, m_new);
      m[0] = m_new;
      l[0] = l[0] * f + x.y * g;
      o[0].x = o[0].x * f + x.z * g;
      o[0].y = o[0].y * f + x.w * g;
    }
  }
  if (lane_has)
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h >= heads) break;
      const bool empty = n == 0;
      const float inv = a.out_scale / l[h];
      const int64_t at = ((int64_t)r * a.Hq + g * a.G + h0 + h) * D + 2 * lane;
      const float x = empty ? 0.f : o[h].x * inv, y = empty ? 0.f : o[h].y * inv;
      if (a.out_bf16) *(unsigned*)((unsigned short*)a.out + at) = (unsigned)float_to_bf16_bits(x) | ((unsigned)float_to_bf16_bits(y) << 16);
      else *(float2*)((float*)a.out + at) = make_float2(x, y);
    }
}

}  // namespace
