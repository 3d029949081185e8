// What a model says of its tokens, from a row of logits read once: log-probability of a given token and how many logits are larger, the
// entropy, and the n_top largest with their log-probabilities.
//
//   m = max x,  l = sum e^(x - m),  t = sum e^(x - m) (x - m):   log p_i = x_i - m - ln l,   H = ln l - t / l     (x: scaled logits)
//
// A lane keeps (m, l, t) of what it has read and rescales when its maximum rises; states are joined as softmax states are.
//
// The largest: a logit and its token make one key (the logit's bits in an order that whole numbers have too, then the token,
// smaller ones larger), so that no two are equal and the result does not depend on any order of work.  The 64 lanes' running maxima
// are maxima of 64 sets that share nothing, so the n_top-th largest of them bounds the n_top-th largest logit from below, and it is a
// good bound: of 128 000 random ones about 24 are above it for 20.  Logits above the bound are kept in LDS, the bound is
// renewed as a wave has read 4, 16, 64 times as much, and at the end those that are left are ranked by counting.  A list that
// fills up all the same (ascending rows, equal ones) is cut down to its n_top largest, whose last is a bound too.
//
// Bound by memory for many rows.  Few rows are cut into parts, a work-group each, whose states and largest a second launch joins.
#pragma once

#include "kernels_common.h"

namespace {

constexpr int SCORE_PARTS = 64;             // most parts of a row: a lane each in the joining launch
constexpr int SCORE_KEPT = 256;             // keys that a wave keeps
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
// Adds another state; a part that is 0 in the sum adds nothing (its t may be beyond all numbers by then).
__device__ __forceinline__ void join(ScoreState& a, const ScoreState& b, float scale_log2) {
  const float m = fmaxf(a.m, b.m), da = a.m - m, db = b.m - m;
  const float fa = __builtin_amdgcn_exp2f(da * scale_log2), fb = __builtin_amdgcn_exp2f(db * scale_log2);
  const float ta = fa == 0.f || a.l == 0.f ? 0.f : fa * (a.t + a.l * da), tb = fb == 0.f || b.l == 0.f ? 0.f : fb * (b.t + b.l * db);
  a.t = ta + tb;
  a.l = (fa == 0.f && a.l == a.l ? 0.f : a.l * fa) + (fb == 0.f && b.l == b.l ? 0.f : b.l * fb);
  a.m = m;
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

// The largest number with BITS leading bits (zeros behind) that at least k of the wave's N x 64 numbers reach.
template <int BITS, int N>
__device__ __forceinline__ unsigned reached_by(const unsigned (&v)[N], int k) {
  unsigned found = 0;
#pragma unroll 1
  for (int bit = 31; bit > 31 - BITS; --bit) {
    const unsigned tried = found | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += count_of(__builtin_amdgcn_ballot_w64(v[i] >= tried));
    if (n >= k) found = tried;
  }
  return found;
}

// Ranks the keys of a list in LDS by counting: `put(rank, key)` for the n_top largest, and for key 0 where there are fewer.
template <typename Put>
__device__ __forceinline__ void rank_keys(const u64* list, int n, int n_top, Put put) {
  for (int i = threadIdx.x; i < n; i += 256) {
    const u64 key = list[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += list[j] > key;
    if (r < n_top) put(r, key);
  }
  for (int r = n + threadIdx.x; r < n_top; r += 256) put(r, (u64)0);
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

// A work-group of four waves for each part of each row.
template <typename T>
__global__ __launch_bounds__(256) void score_kernel(ScoreArgs a) {
  constexpr int V = 16 / (int)sizeof(T), U = 4;              // elements of a piece; pieces of a lane that are loaded together
  constexpr int BITS = sizeof(T) == 2 ? 16 : 20;             // of a bound
  __shared__ u64 kept[4][SCORE_KEPT];
  __shared__ u64 list[4 * SCORE_KEPT];
  __shared__ float lane_max[4][64];
  __shared__ ScoreState states[4];
  __shared__ u64 bounds[4];
  __shared__ int larger_of[4], listed;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x / a.parts;
  const int part = (int)((int64_t)blockIdx.x - row * a.parts);
  if (!row_there(a, row)) return;
  const T* p = (const T*)a.logits + row * a.stride;
  const int e0 = part * a.part_len, e1 = min(e0 + a.part_len, a.vocab);
  const int token = a.tokens ? a.tokens[row] : ODMA_TOKEN_NONE;
  const float given = token >= 0 && token < a.vocab ? score_element(p + token) : __builtin_nanf("");
  lane_max[wave][lane] = LOWEST_REF;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  // whole pieces, and up to 2 V - 2 elements in front of and behind them
  const int lead = min((int)((16 - ((uintptr_t)(p + e0) & 15)) & 15) / (int)sizeof(T), e1 - e0);
  const int pieces = (e1 - e0 - lead) / V, body = e0 + lead, tail = body + pieces * V;
  ScoreState s{LOWEST_REF, 0.f, 0.f};
  int larger = 0, held = 0;
  u64 bound = (u64)ORDERED_OFF << 32 | 0xffffffffu;          // keys above it are kept
  float least = -INFINITY;                                   // what is not above it cannot be among them

  auto set_bound = [&](u64 b) {
    if (b <= bound) return;
    bound = b;
    const unsigned v = (unsigned)(b >> 32);
    least = v <= ORDERED_OFF + 2 ? -INFINITY : of_ordered(v - 2);   // (a step more than is needed: -0 stands between 0 and what is below it)
  };
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
      if (keep) kept[wave][n + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0))] = key[i];
      n += count_of(mask);
    }
    held = n;
    set_bound(found);
  };
  // the statistics of a piece; returns its largest
  auto add = [&](const float* x, int n) {
    float most = x[0];
    for (int i = 1; i < n; ++i) most = fmaxf(most, x[i]);
    if (most > s.m) {
      const float d = s.m - most, f = __builtin_amdgcn_exp2f(d * a.scale_log2);
      s.t = f == 0.f ? 0.f : f * (s.t + s.l * d);
      s.l = f == 0.f && s.l == s.l ? 0.f : s.l * f;
      s.m = most;
    }
    for (int i = 0; i < n; ++i) {
      const float d = x[i] - s.m, e = __builtin_amdgcn_exp2f(d * a.scale_log2);
      s.l += e;
      s.t = __builtin_fmaf(e, fmaxf(d, LOWEST_REF), s.t);    // (0 x -inf)
    }
    if (most > given)
      for (int i = 0; i < n; ++i) larger += x[i] > given;
    return most;
  };
  auto collect = [&](const float* x, int n, float most, int at) {
    if (!__builtin_amdgcn_ballot_w64(most > least)) return;
    for (int i = 0; i < n; ++i) {
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
      if (keep) kept[wave][held + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0))] = key;
      held += count_of(mask);
    }
  };
  // a bound from all lanes' maxima so far (of other waves: as of some moment before, a bound too)
  auto renew = [&]() {
    __hip_atomic_store(&lane_max[wave][lane], s.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    unsigned most[1] = {0};
#pragma unroll
    for (int w = 0; w < 4; ++w)
      most[0] = max(most[0], ordered(w == wave ? s.m : __hip_atomic_load(&lane_max[w][lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)));
    set_bound((u64)reached_by<BITS>(most, a.n_top) << 32);
  };

  int round = 0;
  for (int g = wave * 64; g < pieces; g += 256 * U, ++round) {
    uint4v w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = g + u * 256 + lane;
      w[u] = uint4v{0, 0, 0, 0};
      if (i < pieces) w[u] = *(const uint4v*)(p + body + i * V);
    }
    float x[U][V], most[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      score_piece((const T*)nullptr, w[u], x[u]);
      if (g + u * 256 + lane >= pieces)
#pragma unroll
        for (int i = 0; i < V; ++i) x[u][i] = -INFINITY;
      most[u] = add(x[u], V);
    }
    if (a.n_top > 0) {
      if ((round & (round - 1)) == 0 && (round & 0x55555555 || round == 0)) renew();   // rounds 0, 1, 4, 16, ...
#pragma unroll
      for (int u = 0; u < U; ++u) collect(x[u], V, most[u], body + (g + u * 256 + lane) * V);
    }
  }
  if (wave == 3 && lead + e1 - tail > 0) {                   // single elements
    const int at = lane < lead ? e0 + lane : tail + lane - lead;
    float x[1] = {at < e1 ? score_element(p + at) : -INFINITY};
    const float most = add(x, 1);
    if (a.n_top > 0) collect(x, 1, most, at);
  }
  // ---- the waves together
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    // (lane_max of this wave as it ends; s itself is joined over the lanes)
    if (o == 32) lane_max[wave][lane] = s.m;
    const ScoreState other{__shfl_xor(s.m, o), __shfl_xor(s.l, o), __shfl_xor(s.t, o)};
    join(s, other, a.scale_log2);
    larger += __shfl_xor(larger, o);
  }
  if (lane == 0) {
    states[wave] = s;
    larger_of[wave] = larger;
    bounds[wave] = bound;
  }
  __syncthreads();
  s = states[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) join(s, states[w], a.scale_log2);
  larger = larger_of[0] + larger_of[1] + larger_of[2] + larger_of[3];
  if (threadIdx.x == 0) {
    if (a.parts == 1) put_row(a, row, s, token, given, larger);
    else a.part_state[row * a.parts + part] = make_float4(s.m, s.l, s.t, __int_as_float(larger));
  }
  if (a.n_top == 0) return;
  {
    unsigned most[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) most[w] = ordered(lane_max[w][lane]);
    u64 b = (u64)reached_by<BITS>(most, a.n_top) << 32;
#pragma unroll
    for (int w = 0; w < 4; ++w) b = max(b, bounds[w]);
    for (int i = lane; i < (held + 63) / 64 * 64; i += 64) {
      const u64 key = i < held ? kept[wave][i] : 0;
      const bool keep = key >= b;                            // (a bound may be a key that is kept)
      const u64 mask = __builtin_amdgcn_ballot_w64(keep);
      int from = 0;
      if (lane == 0 && mask) from = atomicAdd(&listed, count_of(mask));
      from = rfl(from);
      if (keep) list[from + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0))] = key;
    }
  }
  __syncthreads();
  const float log_l = log_of(s.l);
  rank_keys(list, listed, a.n_top, [&](int r, u64 key) {
    if (a.parts == 1) put_top(a, row, s, log_l, r, key);
    else a.part_key[(row * a.parts + part) * a.n_top + r] = key;
  });
}

// The parts of a row: a work-group each.
__global__ __launch_bounds__(256) void score_join_kernel(ScoreArgs a) {
  __shared__ u64 list[SCORE_PARTS * ODMA_MAX_ALTERNATIVES];
  __shared__ int listed;
  const int lane = threadIdx.x & 63;
  const int64_t row = blockIdx.x;
  if (!row_there(a, row)) return;
  if (threadIdx.x == 0) listed = 0;
  ScoreState s{LOWEST_REF, 0.f, 0.f};
  int larger = 0;
  if (lane < a.parts) {
    const float4 v = a.part_state[row * a.parts + lane];
    s = ScoreState{v.x, v.y, v.z};
    larger = __float_as_int(v.w);
  }
  const u64* keys = a.part_key + row * a.parts * a.n_top;
  // every part's j-th largest: the q-th largest of those has j q >= n_top keys that reach it
  const int j = a.n_top ? (2 * a.n_top + a.parts - 1) / a.parts : 0, q = j ? (a.n_top + j - 1) / j : 0;
  const int at = min(j, a.n_top);
  unsigned head[1] = {a.n_top && lane < a.parts ? (unsigned)(keys[lane * a.n_top + at - 1] >> 32) : 0u};
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const ScoreState other{__shfl_xor(s.m, o), __shfl_xor(s.l, o), __shfl_xor(s.t, o)};
    join(s, other, a.scale_log2);
    larger += __shfl_xor(larger, o);
  }
  if (threadIdx.x == 0) {
    const int token = a.tokens ? a.tokens[row] : ODMA_TOKEN_NONE;
    float given = 0.f;
    if (token >= 0 && token < a.vocab) given = a.logits_f32 ? ((const float*)a.logits)[row * a.stride + token] : bf16_bits_to_float(((const unsigned short*)a.logits)[row * a.stride + token]);
    put_row(a, row, s, token, given, larger);
  }
  if (a.n_top == 0) return;
  const u64 bound = (u64)reached_by<32>(head, q) << 32;
  __syncthreads();
  for (int i = threadIdx.x; i < a.parts * a.n_top; i += 256) {
    const u64 key = keys[i];
    if (key > bound) list[atomicAdd(&listed, 1)] = key;      // (a bound has no token behind it: keys that reach it are above it)
  }
  __syncthreads();
  const float log_l = log_of(s.l);
  rank_keys(list, listed, a.n_top, [&](int r, u64 key) { put_top(a, row, s, log_l, r, key); });
}

}  // namespace
