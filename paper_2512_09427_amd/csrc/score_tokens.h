// What a model says of its tokens, from a row of logits read once: log-probability of a given token and how many logits are larger, the
// entropy, and the n_top largest with their log-probabilities.
//
//   m = max x,  l = sum e^(x - m),  t = sum e^(x - m) (x - m):   log p_i = x_i - m - ln l,   H = ln l - t / l     (x: scaled logits)
//
// A lane keeps (m, l, t) of what it has read and rescales when its maximum rises; states are joined as softmax states are.
//
// The largest: a logit and its token make one key (the logit's bits in an order that whole numbers have too, then the token,
// smaller ones larger), so that no two are equal and the result does not depend on any order of work.  The lanes' running maxima
// are maxima of sets that share nothing, so the n_top-th largest of them bounds the n_top-th largest logit from below, and it is a
// good bound: of random logits about 24 are above the 20th of 64 maxima, 74 above the 64th of 256.  Logits above the bound are kept
// in LDS, the bound is renewed as a row's read part doubles, and in the end those that are left are ranked by counting.  A list
// that fills up all the same (ascending rows, equal ones) is cut down to its n_top largest, whose last is a bound too.
//
// Bound by memory for many rows (4 096 rows of 50 001 in fp32 5.9 TB/s, in bf16, where a byte brings twice the work, 5.1 to 5.3).  Few long rows are
// cut into parts, a work-group each, whose states and largest a second launch joins.
#pragma once

#include "kernels_common.h"
#include "wave_reduce.h"

namespace {

constexpr int SCORE_PARTS = 64;             // most parts of a row: a lane each in the joining launch
constexpr int SCORE_KEPT = 128;             // keys that a wave keeps: a list that is cut down, and what 64 lanes may add
constexpr int SCORE_RANKED = 128;           // keys that are ranked without another bound
constexpr int SCORE_FAR_LOG2 = 28;          // scaled logits up to 2^28 either way have a rounded reference
constexpr float SCORE_SLACK = 8.f;
typedef unsigned long long u64;

struct ScoreArgs {
  const void* logits;
  int64_t stride, n_rows, pool_tokens;
  const int32_t* tokens;
  const int64_t* row_slot;
  float *logprob, *entropy, *top_logprob;
  int32_t *rank, *top_id;
  float4* part_state;                        // [row][part] m, l, t, how many are larger
  u64* part_key;                             // [row][part][n_top], largest first, 0 behind them
  int32_t vocab, n_top, parts, part_len;     // elements of a part
  int32_t logits_f32;
  float scale, scale_log2;
  float far;                                 // a power of two: far * scale_log2 is exact and at most 2^SCORE_FAR_LOG2
};

// Floats as whole numbers in the same order; 0 and -0 are one.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned b = __float_as_uint(x + 0.f);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_ordered(unsigned u) { return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u); }
constexpr unsigned ORDERED_OFF = 0x007fffffu;                // of -inf
__device__ __forceinline__ u64 score_key(float x, int token) { return (u64)ordered(x) << 32 | (unsigned)~token; }
__device__ __forceinline__ int count_of(u64 mask) { return __builtin_popcountll(mask); }

struct ScoreState {
  float m, l, t;
};
// A product that is rounded by itself, whatever it is subtracted from.
__device__ __forceinline__ float rounded_product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}
// The states of a wave's lanes together, in all of them.  One that is 0 in the sum adds nothing (its t may be beyond all numbers by then), and one of no
// tokens has no say in the reference, which may be above all tokens that others have.
__device__ __forceinline__ ScoreState join_lanes(const ScoreState& s, float scale_log2) {
  const float m = max_over_wave(s.l == 0.f ? LOWEST_REF : s.m), d = s.m - m, f = __builtin_amdgcn_exp2f(d * scale_log2);
  const bool none = (f == 0.f && s.l == s.l) || s.l == 0.f;
  return ScoreState{m, sum_over_wave(none ? 0.f : s.l * f), sum_over_wave(none ? 0.f : f * (s.t + s.l * d))};
}

__device__ __forceinline__ float score_element(const unsigned short* p) { return bf16_bits_to_float(*p); }
__device__ __forceinline__ float score_element(const float* p) { return *p; }
__device__ __forceinline__ void score_piece(const unsigned short*, uint4v w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void score_piece(const float*, uint4v w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
}

// The largest number with BITS leading bits (an even number of them, zeros behind) that at least k of the wave's N x 64 numbers reach: two bits
// at a time, three counts that do not wait for one another.
template <int BITS, int N>
__device__ __forceinline__ unsigned reached_by(const unsigned (&v)[N], int k) {
  unsigned found = 0;
#pragma unroll
  for (int bit = 30; bit > 30 - BITS; bit -= 2) {
    int n[3] = {0, 0, 0};
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < N; ++i) n[t] += count_of(__builtin_amdgcn_ballot_w64(v[i] >= (found | (unsigned)(t + 1) << bit)));
    const unsigned more = n[2] >= k ? 3 : n[1] >= k ? 2 : n[0] >= k ? 1 : 0;
    found |= more << bit;
  }
  return found;
}

// Ranks the keys of a list in LDS by counting, four lanes a key: `put(rank, key)` for the n_top largest, and for key 0 where there are fewer.
template <int THREADS, typename Put>
__device__ __forceinline__ void rank_keys(const u64* list, int n, int n_top, Put put) {
  const int quarter = threadIdx.x & 3;
  for (int i = threadIdx.x >> 2; i < n; i += THREADS / 4) {
    const u64 key = list[i];
    unsigned r = 0;
    int j = quarter;
    for (; j + 28 < n; j += 32) {
      u64 other[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) other[e] = list[j + 4 * e];
#pragma unroll
      for (int e = 0; e < 8; ++e) r += other[e] > key;
    }
#pragma unroll 1
    for (; j < n; j += 4) r += list[j] > key;
    r += moved<0xb1>(r);                                     // of the four lanes
    r += moved<0x4e>(r);
    if (quarter == 0 && r < (unsigned)n_top) put((int)r, key);
  }
  for (int r = n + threadIdx.x; r < n_top; r += THREADS) put(r, (u64)0);
}

// The results of a row, from its whole state.
__device__ __forceinline__ float log_of(float l) { return 0.69314718055994531f * __builtin_amdgcn_logf(l); }
__device__ __forceinline__ float logprob_of(const ScoreArgs& a, const ScoreState& s, float x, float log_l) {
  return s.l == 0.f ? -INFINITY : 2.f * (a.scale * (0.5f * x - 0.5f * s.m)) - log_l;   // (halves: a difference may be beyond fp32 before it is scaled)
}
__device__ __forceinline__ void put_row(const ScoreArgs& a, int64_t row, const ScoreState& s, int token, float x, int larger) {
  const float log_l = log_of(s.l);
  const bool real = token >= 0 && token < a.vocab;
  if (a.logprob) a.logprob[row] = real ? logprob_of(a, s, x, log_l) : -INFINITY;
  if (a.rank) a.rank[row] = real ? larger : a.vocab;
  if (a.entropy) a.entropy[row] = s.l == 0.f ? 0.f : log_l - a.scale * (s.t / s.l);
}
__device__ __forceinline__ void put_top(const ScoreArgs& a, int64_t row, const ScoreState& s, float log_l, int r, u64 key) {
  const float x = key ? of_ordered((unsigned)(key >> 32)) : -INFINITY;
  if (a.top_id) a.top_id[row * a.n_top + r] = key ? (int)~(unsigned)key : ODMA_TOKEN_NONE;
  if (a.top_logprob) a.top_logprob[row * a.n_top + r] = key ? logprob_of(a, s, x, log_l) : -INFINITY;
}

__device__ __forceinline__ bool row_there(const ScoreArgs& a, int64_t row) {
  if (!a.row_slot) return true;
  const int64_t slot = a.row_slot[row];
  return slot != ODMA_SLOT_NONE && slot < a.pool_tokens;
}

// A work-group of W waves for each part of each row.
template <typename T, int W>
__global__ __launch_bounds__(W * 64) void score_kernel(ScoreArgs a) {
  constexpr int V = 16 / (int)sizeof(T), U = 4;              // elements of a piece; pieces of a lane that are loaded together
  constexpr int N = W * 64;                                  // lanes
  constexpr int BITS = sizeof(T) == 2 ? 16 : 20;             // of a bound
  __shared__ u64 kept[W][SCORE_KEPT];
  __shared__ u64 list[W * SCORE_KEPT];
  __shared__ float lane_max[W][64];
  __shared__ ScoreState states[W];
  __shared__ u64 best;                                       // of the waves' bounds
  __shared__ float tops[W];
  __shared__ int larger_of[W], held_of[W], listed;
  const int lane = threadIdx.x & 63, wave = rfl(threadIdx.x >> 6);
  const int64_t row = (int64_t)blockIdx.x / a.parts;
  const int part = (int)((int64_t)blockIdx.x - row * a.parts);
  if (!row_there(a, row)) return;
  const T* p = (const T*)a.logits + row * a.stride;
  const int e0 = part * a.part_len, e1 = min(e0 + a.part_len, a.vocab);
  const int token = a.tokens ? a.tokens[row] : ODMA_TOKEN_NONE;
  // whole pieces, and up to 2 V - 2 elements in front of and behind them
  const int lead = min((int)((16 - ((uintptr_t)(p + e0) & 15)) & 15) / (int)sizeof(T), e1 - e0);
  const int pieces = (e1 - e0 - lead) / V, body = e0 + lead, tail = body + pieces * V;
  uint4v w[U] = {};
  auto load = [&](int g) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (g + u * N >= pieces) continue;
      w[u] = __builtin_nontemporal_load((const uint4v*)(p + body) + min(g + u * N + lane, pieces - 1));
    }
  };
  load(wave * 64);                                           // under way while the given token's logit is looked up
  if (threadIdx.x == 0) {
    listed = 0;
    best = 0;
  }
  const float given = token >= 0 && token < a.vocab ? score_element(p + token) : __builtin_nanf("");
  // The lane's state, in powers of two and with a rounded reference: l = sum 2^(c x - r), t = sum 2^(c x - r) (c x - r), c x - r in one rounding.
  // That rounding is half a step of r, and no term is farther from its value than by a power of it: 2^8 as long as r is within 2^28, while from 2^31 on it
  // would leave fp32.  So the reference starts at a logit of -far, which lower ones (a mask of -1e9) leave as it is, and rows whose largest
  // logit is not between -far and far are taken again below.
  // It moves when a logit is 2^SCORE_SLACK times likelier: of 64 lanes one finds a new largest logit in nearly every piece.
  const float c = a.scale_log2, slack = SCORE_SLACK / c;
  float m = -a.far, raise = m, r = rounded_product(m, c), l = 0.f, t = 0.f, top = -INFINITY;    // (top: the largest as it is)
  int larger = 0, held = 0, round = 0;
  u64 bound = (u64)ORDERED_OFF << 32 | 0xffffffffu;          // keys above it are kept
  float least = -INFINITY;                                   // what is not above it cannot be among them

  auto set_bound = [&](u64 b) {
    if (b <= bound) return;
    bound = b;
    const unsigned v = (unsigned)(b >> 32);
    least = v <= ORDERED_OFF + 2 ? -INFINITY : of_ordered(v - 2);   // (a step more than is needed: -0 stands between 0 and what is below it)
  };
  auto behind = [](u64 mask) { return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0)); };
  // The list cut down to its n_top largest
  auto cut = [&]() {
    u64 key[SCORE_KEPT / 64];
#pragma unroll
    for (int i = 0; i < SCORE_KEPT / 64; ++i) key[i] = i * 64 + lane < held ? kept[wave][i * 64 + lane] : 0;
    u64 found = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const u64 tried = found | 1ull << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < SCORE_KEPT / 64; ++i) n += count_of(__builtin_amdgcn_ballot_w64(key[i] >= tried));
      if (n >= a.n_top) found = tried;
    }
    int n = 0;
#pragma unroll
    for (int i = 0; i < SCORE_KEPT / 64; ++i) {
      const bool keep = key[i] >= found && key[i] != 0;
      const u64 mask = __builtin_amdgcn_ballot_w64(keep);
      if (keep) kept[wave][n + behind(mask)] = key[i];
      n += count_of(mask);
    }
    held = n;
    set_bound(found);
  };
  // the statistics of a piece; returns its largest
  auto add = [&](const float* x, int n) {
    float most = x[0];
    for (int i = 1; i < n; ++i) most = fmaxf(most, x[i]);
    if (most > raise) {
      m = most;
      raise = most + slack;
      const float now = rounded_product(m, c), d = r - now, f = __builtin_amdgcn_exp2f(d);
      t = f == 0.f ? 0.f : f * __builtin_fmaf(l, d, t);
      l *= f;
      r = now;
    }
    for (int i = 0; i < n; ++i) {
      const float d = __builtin_fmaf(x[i], c, -r), e = __builtin_amdgcn_exp2f(d);
      l += e;
      t = __builtin_fmaf(e, fmaxf(d, LOWEST_REF), t);        // (0 x -inf)
    }
    top = most > top ? most : top;
    return most;
  };
  auto count = [&](const float* x, int n, float most) {       // (of the whole wave)
    if (!__builtin_amdgcn_ballot_w64(most > given)) return;
    for (int i = 0; i < n; ++i) larger += count_of(__builtin_amdgcn_ballot_w64(x[i] > given));
  };
  auto collect = [&](const float* x, int n, float most, int at) {
    if (!__builtin_amdgcn_ballot_w64(most > least)) return;
    for (int i = 0; i < n; ++i) {
      if (!__builtin_amdgcn_ballot_w64(x[i] > least)) continue;
      const u64 key = score_key(x[i], at + i);
      bool keep = x[i] > least && key > bound;
      u64 mask = __builtin_amdgcn_ballot_w64(keep);
      if (!mask) continue;
      if (held + count_of(mask) > SCORE_KEPT) {
        __builtin_amdgcn_wave_barrier();
        cut();
        __builtin_amdgcn_wave_barrier();
        keep = keep && key > bound;
        mask = __builtin_amdgcn_ballot_w64(keep);
      }
      if (keep) kept[wave][held + behind(mask)] = key;
      held += count_of(mask);
    }
  };
  auto publish = [&]() { __hip_atomic_store(&lane_max[wave][lane], top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); };
  // a bound from all lanes' maxima (of other waves: as of some moment since they published, which bounds too): 64 sets, or 256 where many
  // are looked for
  auto renew = [&]() {
    unsigned most[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < W; ++i)
      most[i % 4] = max(most[i % 4], ordered(__hip_atomic_load(&lane_max[i][lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)));
    const unsigned one[1] = {(unsigned)max(max(most[0], most[1]), max(most[2], most[3]))};
    set_bound((u64)(a.n_top <= 24 ? reached_by<BITS>(one, a.n_top) : reached_by<BITS>(most, a.n_top)) << 32);
  };

  bool first = true;
  for (int g = wave * 64; g < pieces || first; g += N * U, ++round) {
    float x[U][V], most[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      score_piece((const T*)nullptr, w[u], x[u]);
      if (g + u * N + 64 > pieces) {                         // (the whole wave)
        asm volatile("" ::: "memory");                       // (or the compiler makes 8 moves of it that every piece goes through)
        if (g + u * N + lane >= pieces)
#pragma unroll
          for (int i = 0; i < V; ++i) x[u][i] = -INFINITY;
      }
    }
    load(g + N * U);                                         // under way while these are taken in
#pragma unroll
    for (int u = 0; u < U; ++u) {
      most[u] = -INFINITY;
      if (g + u * N < pieces) most[u] = add(x[u], V);
    }
    if (a.n_top > 0) {
      if ((round & (round + 1)) == 0) {                      // rounds 0, 1, 3, 7, ...
        publish();
        if (first) __syncthreads();
        renew();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) collect(x[u], V, most[u], body + (g + u * N + lane) * V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) count(x[u], V, most[u]);
    first = false;
  }
  if (wave == W - 1 && lead + e1 - tail > 0) {               // single elements
    const int at = lane < lead ? e0 + lane : tail + lane - lead;
    float x[1] = {at < e1 ? score_element(p + at) : -INFINITY};
    const float most = add(x, 1);
    if (a.n_top > 0) collect(x, 1, most, at);
    count(x, 1, most);
  }
  // ---- the waves together.  The power of the reference m is off from r by the rounding of r
  const float d = __builtin_fmaf(m, c, -r), f = __builtin_amdgcn_exp2f(-d);
  ScoreState s = join_lanes(ScoreState{m, l * f, f * __builtin_fmaf(-d, l, t) / c}, c);
  publish();
  top = max_over_wave(top);
  if (lane == 0) {
    states[wave] = s;
    tops[wave] = top;
    larger_of[wave] = larger;
    held_of[wave] = held;
    if (a.n_top > 0) atomicMax(&best, bound);
  }
  __syncthreads();
  auto of_waves = [&]() { return join_lanes(lane < W ? states[lane] : ScoreState{LOWEST_REF, 0.f, 0.f}, c); };   // a wave's state a lane
  s = of_waves();
  top = max_over_wave(lane < W ? tops[lane] : -INFINITY);
  larger = (int)sum_over_wave(lane < W ? (unsigned)larger_of[lane] : 0u);
  const int total = (int)sum_over_wave(lane < W ? (unsigned)held_of[lane] : 0u);
  if (top > a.far || (top <= -a.far && top > -INFINITY)) {   // (the whole work-group) element by element, by differences
    s = ScoreState{LOWEST_REF, 0.f, 0.f};
    for (int i = e0 + threadIdx.x; i < e1; i += N) {
      const float x = score_element(p + i), most = fmaxf(x, s.m);
      const float rise = s.m - most, fall = fmaxf(x - most, LOWEST_REF), e = __builtin_amdgcn_exp2f((x - most) * c);
      const float f = __builtin_amdgcn_exp2f(rise * c);
      s.t = (f == 0.f ? 0.f : f * (s.t + s.l * rise)) + e * fall;
      s.l = (f == 0.f && s.l == s.l ? 0.f : s.l * f) + e;
      s.m = most;
    }
    s = join_lanes(s, c);
    __syncthreads();
    if (lane == 0) states[wave] = s;
    __syncthreads();
    s = of_waves();
  }
  if (threadIdx.x == 0) {
    if (a.parts == 1) put_row(a, row, s, token, given, larger);
    else a.part_state[row * a.parts + part] = make_float4(s.m, s.l, s.t, __int_as_float(larger));
  }
  if (a.n_top == 0) return;
  // ---- the largest: what is above every wave's bound, and one of them all where that may be much
  u64 b = best;
  if (total > SCORE_RANKED) {
    renew();
    b = max(b, bound);
  }
  for (int i = lane; i < (held + 63) / 64 * 64; i += 64) {
    const u64 key = i < held ? kept[wave][i] : 0;
    const bool keep = key >= b;                              // (a bound may be a key that is kept)
    const u64 mask = __builtin_amdgcn_ballot_w64(keep);
    int from = 0;
    if (lane == 0 && mask) from = atomicAdd(&listed, count_of(mask));
    from = rfl(from);
    if (keep) list[from + behind(mask)] = key;
  }
  __syncthreads();
  const float log_l = log_of(s.l);
  rank_keys<N>(list, listed, a.n_top, [&](int r, u64 key) {
    if (a.parts == 1) put_top(a, row, s, log_l, r, key);
    else a.part_key[(row * a.parts + part) * a.n_top + r] = key;
  });
}

// The parts of a row together: a work-group for each row.
__global__ __launch_bounds__(256) void score_join_kernel(ScoreArgs a) {
  constexpr int HELD = SCORE_PARTS * ODMA_MAX_ALTERNATIVES / 256;   // keys of a thread
  __shared__ u64 list[SCORE_PARTS * ODMA_MAX_ALTERNATIVES];
  __shared__ int listed;
  const int lane = threadIdx.x & 63;
  const int64_t row = blockIdx.x;
  if (!row_there(a, row)) return;                            // (its logits may not exist)
  // one round of loads: the states, every part's j-th largest, the keys, the given token
  const float4 v = a.part_state[row * a.parts + min(lane, a.parts - 1)];
  const u64* keys = a.part_key + row * a.parts * a.n_top;
  const int n = a.parts * a.n_top;
  // the q-th largest of the parts' j-th has j q >= n_top keys that reach it
  const int j = a.n_top ? (2 * a.n_top + a.parts - 1) / a.parts : 0, q = j ? (a.n_top + j - 1) / j : 0;
  unsigned head[1] = {0};
  if (a.n_top && lane < a.parts) head[0] = (unsigned)(keys[lane * a.n_top + j - 1] >> 32);
  u64 held[HELD];
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (i * 256 >= n) break;
    const int at = i * 256 + threadIdx.x;
    held[i] = at < n ? keys[at] : 0;
  }
  const int token = a.tokens ? a.tokens[row] : ODMA_TOKEN_NONE;
  float given = 0.f;
  if (token >= 0 && token < a.vocab) {
    const int64_t at = row * a.stride + token;
    given = a.logits_f32 ? score_element((const float*)a.logits + at) : score_element((const unsigned short*)a.logits + at);
  }
  if (threadIdx.x == 0) listed = 0;
  ScoreState s{LOWEST_REF, 0.f, 0.f};
  int larger = 0;
  if (lane < a.parts) {
    s = ScoreState{v.x, v.y, v.z};
    larger = __float_as_int(v.w);
  }
  s = join_lanes(s, a.scale_log2);
  larger = (int)sum_over_wave((unsigned)larger);
  if (threadIdx.x == 0) put_row(a, row, s, token, given, larger);
  if (a.n_top == 0) return;
  const u64 bound = (u64)reached_by<32>(head, q) << 32;
  __syncthreads();
  auto add = [&](u64 key) {
    if (key > bound) list[atomicAdd(&listed, 1)] = key;      // (a bound has no token behind it: keys that reach it are above it)
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (i * 256 >= n) break;
    add(held[i]);
  }
  __syncthreads();
  const float log_l = log_of(s.l);
  rank_keys<256>(list, listed, a.n_top, [&](int r, u64 key) { put_top(a, row, s, log_l, r, key); });
}

}  // namespace
