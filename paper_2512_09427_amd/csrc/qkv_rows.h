// Rows between the projections and the attention: for each head a root-mean-square norm of q and k, the rotation by the row's
// positions, q to a dense array and k, v into the pool's blocks.
//
//   y = x / sqrt(mean(x^2) + eps) * w        (per head, if weights are given)
//   (y_i, y_j) -> (y_i cos t - y_j sin t, y_j cos t + y_i sin t),   t = position[axis(f)] * inv_freq[f] for pair f = (i, j)
//
// all in fp32 and rounded once, when the result is stored.  The angle is formed in 64 bits and reduced to a fraction of a turn
// there: in fp32 a position of a million is off by up to 2^-4 of a radian.
//
// Bound by memory, each element read once and written once: 65 869 rows of 28 / 4 heads x 128 in bf16 (1.21 GB) take 240 us, 5.1
// TB/s, where a copy of 1 GiB reaches 5.2; 20 011 rows into fp8 pools with three axes (349 MB) 73 us; one row 5.5 us, a launch
// and three round trips (slots and positions, rows, stores).
//
// A work-group takes 16 consecutive rows, so that a run of tokens fills whole blocks, and a run of heads; GROUP lanes share a head's row, eight channels each: two runs of four that lie where the rotation pairs them, so that every
// pair is inside a lane, cos and sin of its four pairs stay in registers for all heads of the work-group, and a norm is
// log2(GROUP) exchanges.  k and v go through LDS so that they leave as the 16-byte pieces of their blocks.
#pragma once

#include <type_traits>

#include "block_index.h"
#include "kernels_common.h"

namespace {

struct QkvArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;    // elements between rows
  void* q_out;
  const void *q_weight, *k_weight;
  const float* inv_freq;
  const int64_t* row_slot;
  const int32_t* positions;                // [n_axes][n_rows]
  int64_t n_rows, pool_tokens, head_stride;
  char *k_pool, *v_pool;                   // layer base
  float eps, inv_D, k_inv, v_inv;          // 1 / D; fp8: 1 / k_scale, 1 / v_scale
  int32_t Hq, Hkv, D, rot_dim, adjacent;
  int32_t whole, rest, heads_per_wg;       // tiles of 16 rows that a work-group takes whole; others, of which it takes some heads
  uint32_t rest_inverse;                   // 2^32 / rest, upwards (0: rest is 1)
  int32_t stream_q;                        // the queries are more than a cache keeps: they leave past it
  int32_t n_axes;
  alignas(4) uint8_t axis[ODMA_MAX_ROT_PAIRS];
};

// four channels as they lie in memory, and as numbers
struct Bf16x4 {
  uint2v w;
};
struct F32x4 {
  float4v w;
};
__device__ __forceinline__ Bf16x4 take4(const unsigned short* p) { return {*(const uint2v*)p}; }
__device__ __forceinline__ F32x4 take4(const float* p) { return {*(const float4v*)p}; }
__device__ __forceinline__ void widen4(const Bf16x4& r, float* x) {
  x[0] = __uint_as_float(r.w[0] << 16);
  x[1] = __uint_as_float(r.w[0] & 0xffff0000u);
  x[2] = __uint_as_float(r.w[1] << 16);
  x[3] = __uint_as_float(r.w[1] & 0xffff0000u);
}
__device__ __forceinline__ void widen4(const F32x4& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = r.w[i];
}
__device__ __forceinline__ uint2v rounded4(const unsigned short*, const float* x) {
  uint2v w;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = (unsigned)float_to_bf16_bits(x[2 * i]) | ((unsigned)float_to_bf16_bits(x[2 * i + 1]) << 16);
  return w;
}
__device__ __forceinline__ float4v rounded4(const float*, const float* x) { return float4v{x[0], x[1], x[2], x[3]}; }
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* x) {
  *(decltype(rounded4(p, x))*)p = rounded4(p, x);
}
// E4M3, to nearest even; beyond +-448 (infinities too) the largest value, NaN stays NaN
__device__ __forceinline__ float e4m3_range(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }
__device__ __forceinline__ void store4(unsigned char* p, const float* x) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[0]), e4m3_range(x[1]), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[2]), e4m3_range(x[3]), w, true);
  *(int*)p = w;
}

// 1 / sqrt(v); the instruction takes denormal numbers for 0
__device__ __forceinline__ float root_of_inverse(float v) {
  const bool tiny = v < 0x1p-96f;
  return __builtin_amdgcn_rsqf(tiny ? v * 0x1p96f : v) * (tiny ? 0x1p48f : 1.f);
}

// The sum over the GROUP lanes that share a head's row, in all of them: moves inside quads, halves of rows and rows (each leaves its
// lanes with equal sums, so a mirror adds the other half's).
template <int GROUP>
__device__ __forceinline__ float group_sum(float x) {
  auto moved = [](float v, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
  x += moved(x, std::integral_constant<int, 0xb1>{});        // lanes 1 0 3 2
  x += moved(x, std::integral_constant<int, 0x4e>{});        // lanes 2 3 0 1
  if (GROUP >= 8) x += moved(x, std::integral_constant<int, 0x141>{});
  if (GROUP >= 16) x += moved(x, std::integral_constant<int, 0x140>{});
  if (GROUP >= 32) x += __shfl_xor(x, 16);
  return x;
}

// sine and cosine of f turns, |f| <= 1/2: the nearest quarter turn and the Taylor series of what is left, at most an eighth (pi / 4
// radians, where the terms that are left out are below 2^-28 and 2^-30)
__device__ __forceinline__ void sincos_of_turn(float f, float& sn, float& cs) {
  const float quarter = rintf(4.f * f);
  const float t = __builtin_fmaf(-0.25f, quarter, f) * 6.2831853071795865f, t2 = t * t;
  const float s = t * __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float c = __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int k = (int)quarter;                                // (NaN: the series are NaN)
  const float a = k & 1 ? c : s, b = k & 1 ? s : c;
  sn = k & 2 ? -a : a;
  cs = (k + 1) & 2 ? -b : b;
}

// A work-group of 256 threads takes 16 rows of this many heads at a time (32 lanes a head: two rows a thread), and has the loads of a
// few such passes, a batch, in flight together.
constexpr int rows_pass(int group) { return group < 16 ? 16 / group : 1; }
constexpr int rows_batch(int group, int elem_bytes) { return (group > 16 && elem_bytes == 4 ? 2 : 4) * rows_pass(group); }

// T: rows; S: storage of the pools (T, or unsigned char for E4M3).  GROUP: lanes of a head's row, a power of two >= D / 8.
template <typename T, typename S, int GROUP>
__global__ __launch_bounds__(256) void append_qkv_kernel(QkvArgs a) {
  constexpr bool FP8 = sizeof(S) == 1;
  constexpr int X = 16 / (int)sizeof(S);
  constexpr int HP = rows_pass(GROUP);                     // heads of a pass
  constexpr int RP = GROUP > 16 ? GROUP / 16 : 1;          // rows of a thread
  constexpr int HB = rows_batch(GROUP, sizeof(S)), NB = HB / HP;   // heads and passes of a batch
  constexpr int STRIDE = GROUP * 8 + X;                    // staged row, padded: 16 rows' pieces of a channel meet all banks
  __shared__ __attribute__((aligned(16))) S stage[HB * BLK * STRIDE];
  __shared__ int64_t slots[BLK];
  const int tid = threadIdx.x, lane = tid & 63;
  const int u = tid % GROUP, sub = HP > 1 ? tid / (GROUP * BLK) : 0;
  const int row_in = RP > 1 ? tid / GROUP : (tid / GROUP) % BLK;   // (RP = 2: and 8 rows on)
  const int H = a.Hq + 2 * a.Hkv, cut = (int)blockIdx.x - a.whole;   // (cut >= 0: a piece of a tile)
  const int part = cut < 0 ? 0 : a.rest_inverse ? (int)__umulhi((unsigned)cut, a.rest_inverse) : cut;
  const int64_t row0 = (int64_t)(cut < 0 ? (int)blockIdx.x : a.whole + cut - part * a.rest) * BLK;
  const int h0 = part * a.heads_per_wg, h1 = cut < 0 ? H : min(h0 + a.heads_per_wg, H);

  // this lane's channels: [ca, ca + 4) and [cb, cb + 4)
  const bool in_head = u < a.D / 8, turned = 8 * u < a.rot_dim;
  const int ca = a.adjacent || !turned ? 8 * u : 4 * u, cb = a.adjacent || !turned ? 8 * u + 4 : a.rot_dim / 2 + 4 * u;
  int64_t row[RP];
  bool there[RP];                                          // (the row is in the arrays; further down: and has a slot)
#pragma unroll
  for (int rp = 0; rp < RP; ++rp) {
    row[rp] = row0 + row_in + rp * (BLK / RP);
    there[rp] = in_head && row[rp] < a.n_rows;
  }
  // A batch: HB heads of one kind (0: queries, 1: keys, 2: values) from h on, up to end.
  struct Batch {
    int kind, h, end;
  };
  auto batch_at = [&](int head) {                          // head: of all, queries first
    if (head < a.Hq) return Batch{0, head, min(h1, a.Hq)};
    if (head < a.Hq + a.Hkv) return Batch{1, head - a.Hq, min(h1, a.Hq + a.Hkv) - a.Hq};
    return Batch{2, head - a.Hq - a.Hkv, h1 - a.Hq - a.Hkv};
  };
  auto behind = [&](const Batch& b) { return (b.kind > 0 ? a.Hq : 0) + (b.kind > 1 ? a.Hkv : 0) + min(b.h + HB, b.end); };
  using Four = decltype(take4((const T*)nullptr));
  auto load = [&](Four (&x)[NB][RP][2], const Batch& bt) {
    const T* src = (const T*)(bt.kind == 0 ? a.q : bt.kind == 1 ? a.k : a.v);
    const int64_t stride = bt.kind == 0 ? a.q_stride : bt.kind == 1 ? a.k_stride : a.v_stride;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int rp = 0; rp < RP; ++rp) {
        const int hh = bt.h + b * HP + sub;
        x[b][rp][0] = x[b][rp][1] = Four{};
        if (there[rp] && hh < bt.end) {
          const T* p = src + row[rp] * stride + (int64_t)hh * a.D;
          x[b][rp][0] = take4(p + ca);
          x[b][rp][1] = take4(p + cb);
        }
      }
  };

  // ---- one round of loads: the first batch, slots, positions, frequencies, weights (of rows without a slot too).  None waits for
  // another: a row's positions on all axes are loaded beside the axes of the lane's pairs.
  Four next[NB][RP][2];
  Batch bt = batch_at(h0);
  load(next, bt);
  int64_t slot16 = ODMA_SLOT_NONE;
  if (lane < BLK && row0 + lane < a.n_rows) slot16 = a.row_slot[row0 + lane];
  const bool angles = turned && bt.kind < 2;
  int on_axis[RP][ODMA_MAX_AXES];
  float4v freq = {0.f, 0.f, 0.f, 0.f};
  unsigned axes = 0;                                         // of the lane's four pairs, a byte each
  if (angles) {
    if (a.n_axes > 1) axes = *(const unsigned*)(a.axis + 4 * u);
    freq = float4v{a.inv_freq[4 * u], a.inv_freq[4 * u + 1], a.inv_freq[4 * u + 2], a.inv_freq[4 * u + 3]};
  }
#pragma unroll
  for (int rp = 0; rp < RP; ++rp)
#pragma unroll
    for (int ax = 0; ax < ODMA_MAX_AXES; ++ax) on_axis[rp][ax] = ax < a.n_axes && angles && there[rp] ? a.positions[ax * a.n_rows + row[rp]] : 0;
  Four wq4[2], wk4[2];
  const bool norm_q = a.q_weight != nullptr, norm_k = a.k_weight != nullptr;
  wq4[0] = wq4[1] = wk4[0] = wk4[1] = Four{};
  if (in_head && norm_q) {
    wq4[0] = take4((const T*)a.q_weight + ca);
    wq4[1] = take4((const T*)a.q_weight + cb);
  }
  if (in_head && norm_k) {
    wk4[0] = take4((const T*)a.k_weight + ca);
    wk4[1] = take4((const T*)a.k_weight + cb);
  }
  __builtin_amdgcn_sched_barrier(0);
  float cs[RP][4], sn[RP][4];
#pragma unroll
  for (int rp = 0; rp < RP; ++rp)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      cs[rp][e] = 1.f;
      sn[rp][e] = 0.f;
      if (angles) {
        const unsigned ax = axes >> 8 * e & 255;
        const int pos = ax == 0 ? on_axis[rp][0] : ax == 1 ? on_axis[rp][1] : ax == 2 ? on_axis[rp][2] : on_axis[rp][3];
        const double turns = (double)pos * ((double)freq[e] * 0.15915494309189535);
        sincos_of_turn((float)(turns - rint(turns)), sn[rp][e], cs[rp][e]);
      }
    }
  float wq[8], wk[8];
  widen4(wq4[0], wq);
  widen4(wq4[1], wq + 4);
  widen4(wk4[0], wk);
  widen4(wk4[1], wk + 4);

  // ---- the rows' slots: every wave looks at all 16.  A quad is four rows that fill an aligned group of four slots of a block.
  if (slot16 >= a.pool_tokens) slot16 = ODMA_SLOT_NONE;
  unsigned quads, stored;
  {
    bool quad = lane + 3 < BLK && slot16 >= 0 && (slot16 & 3) == 0;
#pragma unroll
    for (int i = 1; i < 4; ++i) quad &= __shfl_down((long long)slot16, i) == slot16 + i;
    quads = (unsigned)__builtin_amdgcn_ballot_w64(quad) & 0xffffu;
    stored = (unsigned)__builtin_amdgcn_ballot_w64(slot16 >= 0) & 0xffffu;
  }
  const unsigned singles = stored & ~(quads | quads << 1 | quads << 2 | quads << 3);
  const unsigned present = (unsigned)__builtin_amdgcn_ballot_w64(slot16 != ODMA_SLOT_NONE) & 0xffffu;
#pragma unroll
  for (int rp = 0; rp < RP; ++rp) there[rp] = there[rp] && (present >> (row_in + rp * (BLK / RP)) & 1);
  if (tid < BLK) slots[tid] = slot16;                        // (read behind the first barrier of keys or values)

  auto prepare = [&](float (&x)[8], const float (&w)[8], bool norm, int rp) {
    if (norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
      const float inv = root_of_inverse(__builtin_fmaf(group_sum<GROUP>(ss), a.inv_D, a.eps));
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * w[i];
    }
    if (turned) {
      if (a.adjacent) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = x[2 * e], z = x[2 * e + 1];
          x[2 * e] = y * cs[rp][e] - z * sn[rp][e];
          x[2 * e + 1] = z * cs[rp][e] + y * sn[rp][e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = x[e], z = x[4 + e];
          x[e] = y * cs[rp][e] - z * sn[rp][e];
          x[4 + e] = z * cs[rp][e] + y * sn[rp][e];
        }
      }
    }
  };
  const int64_t block_bytes = (int64_t)BLK * a.D * (int)sizeof(S);
  const int pieces = a.D / X;                              // 16-byte pieces of a head's row
  for (;;) {
    Four raw[NB][RP][2];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int rp = 0; rp < RP; ++rp)
#pragma unroll
        for (int i = 0; i < 2; ++i) raw[b][rp][i] = next[b][rp][i];
    const int head = behind(bt), h = bt.h, end = bt.end, kv = bt.kind - 1;
    const Batch now = bt;
    if (head < h1) {                                         // under way while this one is prepared and stored
      bt = batch_at(head);
      load(next, bt);
    }
    if (now.kind == 0) {
      // ---- queries
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int rp = 0; rp < RP; ++rp) {
          const int hh = h + b * HP + sub;
          float x[8];
          widen4(raw[b][rp][0], x);
          widen4(raw[b][rp][1], x + 4);
          prepare(x, wq, norm_q, rp);
          if (there[rp] && hh < end) {
            T* o = (T*)a.q_out + (row[rp] * a.Hq + hh) * a.D;
            using Out = decltype(rounded4(o, x));
            const Out lo = rounded4(o, x), hi = rounded4(o, x + 4);
            if (!a.stream_q) {
              *(Out*)(o + ca) = lo;
              *(Out*)(o + cb) = hi;
            } else {
              asm volatile("" ::: "memory");                 // (or the compiler makes ordinary stores of all branches)
              bool whole = false;
              if constexpr (sizeof(T) == 2)
                if (cb == ca + 4) {                          // a store past the caches has to fill what it touches
                  __builtin_nontemporal_store(uint4v{lo[0], lo[1], hi[0], hi[1]}, (uint4v*)(o + ca));
                  whole = true;
                }
              if (!whole) {
                __builtin_nontemporal_store(lo, (Out*)(o + ca));
                __builtin_nontemporal_store(hi, (Out*)(o + cb));
              }
              asm volatile("" ::: "memory");
            }
          }
        }
    } else {
      // ---- keys and values: staged, then written piece by piece
      __syncthreads();                                       // the batch before has been written
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int rp = 0; rp < RP; ++rp) {
          float x[8];
          widen4(raw[b][rp][0], x);
          widen4(raw[b][rp][1], x + 4);
          if (!kv) prepare(x, wk, norm_k, rp);
          if (FP8)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= kv ? a.v_inv : a.k_inv;
          if (in_head) {
            S* o = stage + ((b * HP + sub) * BLK + row_in + rp * (BLK / RP)) * STRIDE;
            store4(o + ca, x);
            store4(o + cb, x + 4);
          }
        }
      __syncthreads();
      const int heads = min(HB, end - h);
      for (int hb = 0; hb < heads; ++hb) {
        const S* rows = stage + hb * BLK * STRIDE;
        char* plane = (kv ? a.v_pool : a.k_pool) + (int64_t)(h + hb) * a.head_stride;
        if (!kv) {
          for (int i = tid; i < BLK * pieces; i += 256) {
            const int t = i & 15, c = i >> 4;
            const int64_t slot = slots[t];
            if (slot < 0) continue;
            char* block = plane + slot / BLK * block_bytes;
            const int at = (int)(slot % BLK);
            if (FP8) {                                     // piece c: channels 64 (c / 4) + 8 (c % 4) .. + 7 and 32 on
              const S* p = rows + t * STRIDE + (c >> 2) * 64 + (c & 3) * 8;
              const uint2v first = *(const uint2v*)p, second = *(const uint2v*)(p + 32);
              *(uint4v*)(block + (c * 16 + at) * 16) = uint4v{first[0], first[1], second[0], second[1]};
            } else {
              *(uint4v*)(block + (c * BLK + at) * 16) = *(const uint4v*)(rows + t * STRIDE + c * X);
            }
          }
        } else {
          // quads: a thread writes four tokens of two channels (fp8: four channels), 16 apart
          constexpr int CG = FP8 ? 4 : 2;                  // channel groups of 16 in a piece
          const int per_quad = a.D / CG;
          for (int i = tid; i < __builtin_popcount(quads) * per_quad; i += 256) {
            const int qi = i / per_quad, e = i - qi * per_quad, c = e & 15, part = e >> 4;   // part: of 16 CG channels
            unsigned left = quads;
            for (int s = 0; s < qi; ++s) left &= left - 1;
            const int t0 = __builtin_ctz(left);
            const int64_t slot = slots[t0];
            char* block = plane + slot / BLK * block_bytes;
            const S* p = rows + t0 * STRIDE + part * 16 * CG + c;
            alignas(16) S piece[4 * CG];
#pragma unroll
            for (int w = 0; w < CG; ++w)
#pragma unroll
              for (int t = 0; t < 4; ++t) piece[4 * w + t] = p[t * STRIDE + 16 * w];
            uint4v* to = (uint4v*)((S*)block + (FP8 ? v_index_fp8((int)(slot % BLK), part * 64 + c) : v_index((int)(slot % BLK), part * 32 + c)));
#pragma unroll
            for (int k = 0; k < (int)sizeof(piece) / 16; ++k) to[k] = ((const uint4v*)piece)[k];
          }
          // other rows: element by element, two rows at a time where their channels leave threads over
          const int rows_at_once = a.D <= 128 ? 2 : 1, half = rows_at_once == 2 ? tid >> 7 : 0, d0 = rows_at_once == 2 ? tid & 127 : tid;
          for (unsigned left = singles; left;) {
            unsigned mine = left;
            left &= left - 1;
            if (rows_at_once == 2) {
              if (half) mine = left;
              left &= left - 1;
            }
            if (!mine || d0 >= a.D) continue;
            const int t = __builtin_ctz(mine);
            const int64_t slot = slots[t];
            S* block = (S*)(plane + slot / BLK * block_bytes);
            block[FP8 ? v_index_fp8((int)(slot % BLK), d0) : v_index((int)(slot % BLK), d0)] = rows[t * STRIDE + d0];
          }
        }
      }
    }
    if (head >= h1) break;
  }
}

}  // namespace
