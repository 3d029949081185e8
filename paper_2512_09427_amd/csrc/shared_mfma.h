// Decode attention of a batch that shares prefixes, for gfx950.
//
// A request's softmax runs over its group's prefix and its own tokens.  Each of the two parts leaves a state of a query
// column (request, query head): reference m, sum l = sum 2^(s - m), O = sum 2^(s - m) V; states join by
//   M = max m_i,  out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i,
// so the prefix can be attended to by the queries of all its requests together: (requests x heads of a KV head's group)
// columns against its tokens, a dense contraction with reuse, where a request by itself only streams.
//
// Two lines of work.  Line A: items (prefix, KV head, block of SHARED_COLS columns), each the pairs of 16-token tiles of the
// prefix.  Line B: items (request, KV head), each the tiles of the request's own tokens.  An item also counts a few units for
// its start and end.  Each line is cut into equal shares, one of each to every work-group, so line A's matrix
// instructions and line B's memory traffic overlap on every compute unit without a number that weighs one against the other: half
// of the work-groups begin with A, half with B.  A share's pieces leave their states in the workspace and
// shared_merge_kernel joins them; where a piece lies follows from the positions on the lines alone.
#pragma once

#include "kernels_common.h"
#include "batch_tables.h"

namespace {

enum { SHARED_BF16_128, SHARED_FP8_128, SHARED_BF16_64 };
constexpr int SHARED_COLS = 128;          // columns of an item of line A: four waves of two 16-column tiles
constexpr int SHARED_CT = 2;
constexpr int SHARED_A_EXTRA = 3;         // start and end of an item of line A, in pairs
constexpr int SHARED_B_EXTRA = 4;         // and of line B, in tiles
constexpr int SHARED_A_LEAST = 8;         // smallest share: pairs and tiles a work-group is given
constexpr int SHARED_B_LEAST = 12;
constexpr int SHARED_MAX_N = ODMA_SHARED_MAX_REQUESTS;
constexpr int SHARED_THREADS = 256;

struct SharedRecord {                     // of a request: where its parts lie on the lines
  int64_t a_pos, b_pos;                   // of the first head's item
  int32_t a_pairs, a_blocks, a_col;       // pairs of the prefix (0: none), column blocks per head, the request's first column
  int32_t b_tiles;
  int64_t a_total, b_total;
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
  int32_t cut_cols;                       // columns kept for the piece that a work-group continues on line A
  SharedRecord* rec;                      // [n]
  float2* part_ml;                        // states of columns: reference and sum
  float* part_o;                          // [column][128]
};

// columns of the workspace: first pieces of line A and of line B by (request, head), then the continued ones by work-group
__device__ __forceinline__ int64_t shared_first(const SharedArgs& a, int line, int r, int hq) {
  return ((int64_t)line * a.n + r) * a.Hq + hq;
}
__device__ __forceinline__ int64_t shared_cut_a(const SharedArgs& a, int w) { return (int64_t)2 * a.n * a.Hq + (int64_t)w * a.cut_cols; }
__device__ __forceinline__ int64_t shared_cut_b(const SharedArgs& a, int w) {
  return (int64_t)2 * a.n * a.Hq + (int64_t)a.workers * a.cut_cols + (int64_t)w * 16;
}

// Shares of a line.  Share w of `used` is [start(w), start(w + 1)); an item at s with T units has unit 0 at s and unit i at
// s + extra + i, and a unit belongs to the share that holds its position.
struct SharedLine {
  int64_t total;
  int used;
  __device__ __forceinline__ SharedLine(int64_t total_, int least, int workers) : total(total_) {
    const int64_t w = total / least;
    used = total == 0 ? 0 : (int)(w < 1 ? 1 : w < workers ? w : workers);
    used = min((used + 7) / 8 * 8, workers);              // every XCD the same number
  }
  __device__ __forceinline__ int64_t start(int w) const { return total * w / used; }
  __device__ __forceinline__ int holder(int64_t pos) const { return (int)(((pos + 1) * used - 1) / total); }
};
// units of an item at s in front of position x
__device__ __forceinline__ int units_before(int64_t x, int64_t s, int T, int extra) {
  if (x <= s) return 0;
  const int64_t i = x - s - extra;
  return (int)(i < 1 ? 1 : i < T ? i : T);
}

template <bool HIGH_HALF>
__device__ __forceinline__ unsigned widen_e4m3x2(unsigned w) {
  typedef float float2v __attribute__((ext_vector_type(2)));
  const float2v f = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HIGH_HALF);
  return (__float_as_uint(f[0]) >> 16) | (__float_as_uint(f[1]) & 0xffff0000u);
}

struct SharedPlan {
  int64_t a_pos[SHARED_MAX_N + 1], b_pos[SHARED_MAX_N + 1];   // exclusive prefix: groups on line A, requests on line B
  int32_t reader[SHARED_MAX_N];                               // of a group: its first request that holds all of the shared part
  int64_t wave_sum[2][SHARED_THREADS / 64];
};

// own tokens of request r (those of its prefix too, where it is shorter than the shared part), and what it shares
struct SharedRequest {
  int len, shared, group;
  __device__ __forceinline__ SharedRequest(const SharedArgs& a, int r) {
    len = max(a.lengths[r], 0);
    group = prefix_of(a.prefix_start, a.n_prefixes, r);
    shared = group >= 0 ? shared_tokens(a.prefix_lengths[group]) : 0;
  }
  __device__ __forceinline__ bool shares() const { return shared > 0 && len >= shared; }
  __device__ __forceinline__ int own() const { return shares() ? len - shared : len; }
};
// members of group p
__device__ __forceinline__ void shared_members(const SharedArgs& a, int p, int& begin, int& count) {
  begin = min(max(a.prefix_start[p], 0), a.n);
  count = max(min(a.prefix_start[p + 1], a.n) - begin, 0);
}
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

// exclusive scan of one value per thread over the work-group; the sum of all in `total`
__device__ __forceinline__ int64_t scan_of_threads(int64_t x, int64_t* wave_sum, int64_t& total) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int64_t inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 63) wave_sum[wv] = inc;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int i = 0; i < SHARED_THREADS / 64; ++i) {
    if (i < wv) before += wave_sum[i];
    total += wave_sum[i];
  }
  return before + inc - x;
}

__device__ __forceinline__ void store_result(const SharedArgs& a, int64_t at, int ch, float x) {
  if (a.out_bf16) ((unsigned short*)a.out)[at + ch] = float_to_bf16_bits(x);
  else ((float*)a.out)[at + ch] = x;
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

  // ---- plan: every work-group for itself (a launch of its own would be one work-group's round trips on an empty chip)
  for (int p = tid; p < a.n_prefixes; p += SHARED_THREADS) plan.reader[p] = a.n;
  __syncthreads();
  const int per = (a.n + SHARED_THREADS - 1) / SHARED_THREADS;
  const int r0 = min(tid * per, a.n), r1 = min(r0 + per, a.n);
  int64_t mine = 0;
  for (int r = r0; r < r1; ++r) {
    const SharedRequest rq(a, r);
    if (rq.shares()) atomicMin(&plan.reader[rq.group], r);
    const int tiles = (int)(((int64_t)rq.own() + BLK - 1) / BLK);
    plan.b_pos[r] = tiles;
    if (tiles) mine += (int64_t)a.Hkv * (tiles + SHARED_B_EXTRA);
  }
  int64_t b_total, a_total;
  int64_t at = scan_of_threads(mine, plan.wave_sum[0], b_total);     // (its barrier: reader is whole)
  for (int r = r0; r < r1; ++r) {
    const int64_t tiles = plan.b_pos[r];
    plan.b_pos[r] = at;
    if (tiles) at += (int64_t)a.Hkv * (tiles + SHARED_B_EXTRA);
  }
  const int perp = (a.n_prefixes + SHARED_THREADS - 1) / SHARED_THREADS;
  const int p0 = min(tid * perp, a.n_prefixes), p1 = min(p0 + perp, a.n_prefixes);
  auto group_cost = [&](int p) -> int64_t {
    int begin, count;
    shared_members(a, p, begin, count);
    const int pairs = (shared_tokens(a.prefix_lengths[p]) / BLK + 1) / 2;
    return plan.reader[p] < a.n ? (int64_t)a.Hkv * column_blocks(count, G) * (pairs + SHARED_A_EXTRA) : 0;
  };
  mine = 0;
  for (int p = p0; p < p1; ++p) mine += group_cost(p);
  at = scan_of_threads(mine, plan.wave_sum[1], a_total);
  for (int p = p0; p < p1; ++p) {
    plan.a_pos[p] = at;
    at += group_cost(p);
  }
  if (tid == 0) {
    plan.a_pos[a.n_prefixes] = a_total;
    plan.b_pos[a.n] = b_total;
  }
  __syncthreads();
  if (blockIdx.x == gridDim.x - 1) {                        // for the merge
    for (int r = tid; r < a.n; r += SHARED_THREADS) {
      const SharedRequest rq(a, r);
      SharedRecord rec = {0, plan.b_pos[r], 0, 0, 0, (int)(((int64_t)rq.own() + BLK - 1) / BLK), a_total, b_total};
      if (rq.shares()) {
        int begin, count;
        shared_members(a, rq.group, begin, count);
        rec.a_pos = plan.a_pos[rq.group];
        rec.a_pairs = (rq.shared / BLK + 1) / 2;
        rec.a_blocks = column_blocks(count, G);
        rec.a_col = (r - begin) * G;
      }
      a.rec[r] = rec;
    }
  }
  const SharedLine la(a_total, SHARED_A_LEAST + SHARED_A_EXTRA, a.workers), lb(b_total, SHARED_B_LEAST + SHARED_B_EXTRA, a.workers);
  // XCD x (work-groups x, x + 8, ..) has neighbouring shares, which read the same heads; a line with few shares takes the first
  // work-groups of every XCD (A) or the last (B).
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, turns = a.workers >> 3;
  const int ja = la.used >> 3, jb = lb.used >> 3;
  const int share_a = turn < ja ? xcd * ja + turn : -1, share_b = turns - 1 - turn < jb ? xcd * jb + turns - 1 - turn : -1;

  auto piece = [&](const uint4v (&w)[LOADS], int s) {       // 16-byte operand s (of NS) of a tile, as bf16
    if (!FP8) return w[s % LOADS];
    const unsigned w0 = w[(s >> 1) % LOADS][2 * (s & 1)], w1 = w[(s >> 1) % LOADS][2 * (s & 1) + 1];
    return uint4v{widen_e4m3x2<false>(w0), widen_e4m3x2<true>(w0), widen_e4m3x2<false>(w1), widen_e4m3x2<true>(w1)};
  };
  auto join = [](uint2v lo, uint2v hi) { return __builtin_bit_cast(bf16x8, uint4v{lo[0], lo[1], hi[0], hi[1]}); };

  // ================= line A
  auto line_a = [&]() {
    const int64_t x0 = la.start(share_a), x1 = la.start(share_a + 1);
    // group that holds x0: the last one at or before it (groups without work repeat a position)
    int lo = 0, hi = a.n_prefixes;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.a_pos[mid] <= x0) lo = mid;
      else hi = mid;
    }
    for (int p = rfl(lo); p < a.n_prefixes && plan.a_pos[p] < x1; ++p) {
      if (plan.a_pos[p + 1] <= x0 || plan.a_pos[p + 1] == plan.a_pos[p]) continue;
      int begin, count;
      shared_members(a, p, begin, count);
      begin = rfl(begin);
      count = rfl(count);
      const int n_tiles = rfl(shared_tokens(a.prefix_lengths[p]) / BLK), pairs = (n_tiles + 1) / 2;
      const int blocks = column_blocks(count, G), cost = pairs + SHARED_A_EXTRA, items = a.Hkv * blocks, n_cols = count * G;
      const int64_t base_pos = plan.a_pos[p];
      const int64_t base_block = PAGED ? 0 : a.prefix_offsets[p] / BLK;
      const const_i32* bt_row = as_constant(PAGED ? a.bt + (int64_t)rfl(plan.reader[p]) * a.bt_stride : nullptr);
      int item = rfl(x0 > base_pos ? (int)((x0 - base_pos) / cost) : 0);
      for (; item < items; ++item) {
        const int64_t s = base_pos + (int64_t)item * cost;
        if (s >= x1) break;
        const int i0 = rfl(units_before(x0, s, pairs, SHARED_A_EXTRA)), i1 = rfl(units_before(x1, s, pairs, SHARED_A_EXTRA));
        if (i0 >= i1) continue;
        const bool continued = x0 > s;
        const int g = rfl(item / blocks), cb = rfl(item - g * blocks);
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
        float m[CT], l[CT];
        float4v O[CT][DT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          m[ct] = LOWEST_REF;
          l[ct] = 0.f;
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
              float4v s4 = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int sp = 0; sp < NS; ++sp) s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[sp], qreg[ct][sp], s4, 0, 0, 0);
              x[ct][b] = s4;
            }
          }
          if (2 * pr + 1 >= n_tiles)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) x[ct][1] = float4v{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          bool move = false;
          float top[CT];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            top[ct] = fmaxf(fmaxf(fmaxf(x[ct][0][0], x[ct][0][1]), fmaxf(x[ct][0][2], x[ct][0][3])),
                            fmaxf(fmaxf(x[ct][1][0], x[ct][1][1]), fmaxf(x[ct][1][2], x[ct][1][3]))) * a.scale_log2;
            move |= top[ct] > m[ct] + SLACK;
          }
          if (__builtin_amdgcn_ballot_w64(move) != 0) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
              top[ct] = fmaxf(top[ct], __shfl_xor(top[ct], 16));
              top[ct] = fmaxf(top[ct], __shfl_xor(top[ct], 32));
              const float m_new = fmaxf(m[ct], top[ct]), f = joined(m[ct], m_new);
              m[ct] = m_new;
              l[ct] *= f;
#pragma unroll
              for (int dt = 0; dt < DT; ++dt) O[ct][dt] *= f;
            }
          }
          bf16x8 ph[CT], pl[CT];
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float pv = __builtin_amdgcn_exp2f(__builtin_fmaf(x[ct][b][i], a.scale_log2, -m[ct]));
                sum += pv;
                if (LO) {
                  __bf16 hi, lo;
                  two_parts(pv, hi, lo);
                  ph[ct][4 * b + i] = hi;
                  pl[ct][4 * b + i] = lo;
                } else {
                  ph[ct][4 * b + i] = (__bf16)pv;
                }
              }
            l[ct] += sum;
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
          l[ct] += __shfl_xor(l[ct], 16);
          l[ct] += __shfl_xor(l[ct], 32);
          if (!ok[ct]) continue;
          const int64_t c = continued ? shared_cut_a(a, share_a) + wv * 16 * CT + 16 * ct + col16 : shared_first(a, 0, row[ct], head[ct]);
          if (g4 == 0) a.part_ml[c] = make_float2(m[ct], l[ct]);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) *(float4v*)(a.part_o + c * 128 + 16 * dt + 4 * g4) = O[ct][dt];
        }
      }
    }
  };

  // ================= line B: one request and KV head at a time; the waves take turns at its pairs of tiles, straight into registers
  auto line_b = [&]() {
    const int64_t x0 = lb.start(share_b), x1 = lb.start(share_b + 1);
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.b_pos[mid] <= x0) lo = mid;
      else hi = mid;
    }
    for (int r = rfl(lo); r < a.n && plan.b_pos[r] < x1; ++r) {
      if (plan.b_pos[r + 1] <= x0 || plan.b_pos[r + 1] == plan.b_pos[r]) continue;
      const SharedRequest rq(a, r);
      const int own = rfl(rq.own()), tiles = (own + BLK - 1) / BLK, cost = tiles + SHARED_B_EXTRA;
      const int in_front = rfl(rq.shares() ? rq.shared / BLK : 0);        // blocks of the row that are not its own
      // its own slab; a request shorter than the shared part reads its group's prefix
      const int64_t base_block = PAGED ? 0 : (rq.shared > 0 && !rq.shares() ? a.prefix_offsets[rq.group] : a.offsets[r]) / BLK;
      const const_i32* bt_row = as_constant(PAGED ? a.bt + (int64_t)r * a.bt_stride + in_front : nullptr);
      const int64_t base_pos = plan.b_pos[r];
      int g = rfl(x0 > base_pos ? (int)((x0 - base_pos) / cost) : 0);
      for (; g < a.Hkv; ++g) {
        const int64_t s = base_pos + (int64_t)g * cost;
        if (s >= x1) break;
        const int i0 = rfl(units_before(x0, s, tiles, SHARED_B_EXTRA)), i1 = rfl(units_before(x1, s, tiles, SHARED_B_EXTRA));
        if (i0 >= i1) continue;
        const bool continued = x0 > s;
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
          float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                            fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3]))) * a.scale_log2;
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
        const int64_t c = continued ? shared_cut_b(a, share_b) : shared_first(a, 1, r, g * G);
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

// Joins the pieces of a request's two parts: a wave per (request, query head), two channels a lane.
template <int D>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t id = rfl(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (id >= (int64_t)a.n * a.Hq) return;
  const int r = (int)(id / a.Hq), hq = (int)(id - (int64_t)r * a.Hq), g = hq / a.G;
  const SharedRecord rec = a.rec[r];
  float m = LOWEST_REF, l = 0.f;
  float2 o = {0.f, 0.f};
  const bool lane_has = 2 * lane < D;
  auto add = [&](int64_t c) {
    const float2 ml = a.part_ml[c];
    const float2 x = lane_has ? *(const float2*)(a.part_o + c * 128 + 2 * lane) : make_float2(0.f, 0.f);
    const float m_new = fmaxf(m, ml.x), f = joined(m, m_new), fx = joined(ml.x, m_new);
    m = m_new;
    l = l * f + ml.y * fx;
    o.x = o.x * f + x.x * fx;
    o.y = o.y * f + x.y * fx;
  };
  if (rec.a_pairs) {
    const SharedLine line(rec.a_total, SHARED_A_LEAST + SHARED_A_EXTRA, a.workers);
    const int col = rec.a_col + hq - g * a.G, cb = col / SHARED_COLS;
    const int64_t s = rec.a_pos + (int64_t)(g * rec.a_blocks + cb) * (rec.a_pairs + SHARED_A_EXTRA);
    int w = line.holder(s);
    add(shared_first(a, 0, r, hq));
    for (int before = units_before(line.start(w + 1), s, rec.a_pairs, SHARED_A_EXTRA); before < rec.a_pairs;) {
      ++w;
      const int upto = units_before(line.start(w + 1), s, rec.a_pairs, SHARED_A_EXTRA);
      if (upto > before) add(shared_cut_a(a, w) + col - cb * SHARED_COLS);   // (a share shorter than an item's start may hold none)
      before = upto;
    }
  }
  if (rec.b_tiles) {
    const SharedLine line(rec.b_total, SHARED_B_LEAST + SHARED_B_EXTRA, a.workers);
    const int64_t s = rec.b_pos + (int64_t)g * (rec.b_tiles + SHARED_B_EXTRA);
    int w = line.holder(s);
    add(shared_first(a, 1, r, hq));
    for (int before = units_before(line.start(w + 1), s, rec.b_tiles, SHARED_B_EXTRA); before < rec.b_tiles;) {
      ++w;
      const int upto = units_before(line.start(w + 1), s, rec.b_tiles, SHARED_B_EXTRA);
      if (upto > before) add(shared_cut_b(a, w) + hq - g * a.G);
      before = upto;
    }
  }
  if (lane_has) {
    const float inv = rec.a_pairs || rec.b_tiles ? a.out_scale / l : 0.f;
    const int64_t at = id * D + 2 * lane;
    const bool empty = !rec.a_pairs && !rec.b_tiles;
    store_result(a, at, 0, empty ? 0.f : o.x * inv);
    store_result(a, at, 1, empty ? 0.f : o.y * inv);
  }
}

}  // namespace
