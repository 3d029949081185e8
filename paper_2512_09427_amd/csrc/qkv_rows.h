// Rows between the projections and the attention: for each head a root-mean-square norm of q and k, the rotation by the row's
// positions, q to a dense array and k, v into the pool's blocks.
//
//   y = x / sqrt(mean(x^2) + eps) * w        (per head, if weights are given)
//   (y_i, y_j) -> (y_i cos t - y_j sin t, y_j cos t + y_i sin t),   t = position[axis(f)] * inv_freq[f] for pair f = (i, j)
//
// all in fp32 and rounded once, when the result is stored.  The angle is formed in 64 bits and reduced to a fraction of a turn
// there: in fp32 a position of a million is off by up to 2^-4 of a radian.
//
// Bound by memory (each element read once and written once).  A work-group takes 16 consecutive rows and a run of heads; GROUP
// lanes share a head's row, eight channels each: two runs of four that lie where the rotation pairs them, so that every
// pair is inside a lane, cos and sin of its four pairs stay in registers for all heads of the work-group, and a norm is
// log2(GROUP) exchanges.  k and v go through LDS so that they leave as the 16-byte pieces of their blocks.
#pragma once

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
  float eps, k_inv, v_inv;                 // fp8: 1 / k_scale, 1 / v_scale
  int32_t Hq, Hkv, D, rot_dim, adjacent, heads_per_wg;
  uint8_t axis[ODMA_MAX_ROT_PAIRS];
};

__device__ __forceinline__ void load4(const unsigned short* p, float (&x)[8], int at) {
  const uint2v w = *(const uint2v*)p;
  x[at] = __uint_as_float(w[0] << 16);
  x[at + 1] = __uint_as_float(w[0] & 0xffff0000u);
  x[at + 2] = __uint_as_float(w[1] << 16);
  x[at + 3] = __uint_as_float(w[1] & 0xffff0000u);
}
__device__ __forceinline__ void load4(const float* p, float (&x)[8], int at) {
  const float4v w = *(const float4v*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[at + i] = w[i];
}
__device__ __forceinline__ void store4(unsigned short* p, const float* x) {
  uint2v w;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = (unsigned)float_to_bf16_bits(x[2 * i]) | ((unsigned)float_to_bf16_bits(x[2 * i + 1]) << 16);
  *(uint2v*)p = w;
}
__device__ __forceinline__ void store4(float* p, const float* x) { *(float4v*)p = float4v{x[0], x[1], x[2], x[3]}; }
// E4M3, to nearest even; beyond +-448 (infinities too) the largest value, NaN stays NaN
__device__ __forceinline__ float e4m3_range(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }
__device__ __forceinline__ void store4(unsigned char* p, const float* x) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[0]), e4m3_range(x[1]), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x[2]), e4m3_range(x[3]), w, true);
  *(int*)p = w;
}

// T: rows; S: storage of the pools (T, or unsigned char for E4M3).  GROUP: lanes of a head's row, a power of two >= D / 8.
template <typename T, typename S, int GROUP>
__global__ __launch_bounds__(256) void append_qkv_kernel(QkvArgs a) {
  constexpr bool FP8 = sizeof(S) == 1;
  constexpr int X = 16 / (int)sizeof(S);
  constexpr int HP = GROUP < 16 ? 16 / GROUP : 1;          // heads of a pass
  constexpr int RP = GROUP > 16 ? GROUP / 16 : 1;          // rows of a thread
  constexpr int NB = GROUP > 16 && sizeof(S) == 4 ? 2 : 4; // passes whose loads are in flight together
  constexpr int HB = NB * HP;                              // heads of a batch
  constexpr int STRIDE = GROUP * 8 + X;                    // staged row, padded: 16 rows' pieces of a channel meet all banks
  __shared__ __attribute__((aligned(16))) S stage[HB * BLK * STRIDE];
  __shared__ int64_t slots[BLK];
  const int tid = threadIdx.x, lane = tid & 63;
  const int u = tid % GROUP, sub = HP > 1 ? tid / (GROUP * BLK) : 0;
  const int row_in = RP > 1 ? tid / GROUP : (tid / GROUP) % BLK;   // (RP = 2: and 8 rows on)
  const int64_t row0 = (int64_t)blockIdx.x * BLK;
  const int H = a.Hq + 2 * a.Hkv, h0 = blockIdx.y * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, H);

  // ---- the rows: every wave looks at all 16.  A quad is four rows that fill an aligned group of four slots of a block.
  int64_t slot16 = ODMA_SLOT_NONE;
  if (lane < BLK && row0 + lane < a.n_rows) slot16 = a.row_slot[row0 + lane];
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
  if (tid < BLK) slots[tid] = slot16;
  __syncthreads();

  // ---- this lane's channels: [ca, ca + 4) and [cb, cb + 4)
  const bool in_head = u < a.D / 8, turned = 8 * u < a.rot_dim;
  const int ca = a.adjacent || !turned ? 8 * u : 4 * u, cb = a.adjacent || !turned ? 8 * u + 4 : a.rot_dim / 2 + 4 * u;
  bool there[RP];
  int64_t row[RP];
  float cs[RP][4], sn[RP][4];
#pragma unroll
  for (int rp = 0; rp < RP; ++rp) {
    row[rp] = row0 + row_in + rp * (BLK / RP);
    there[rp] = in_head && slots[row_in + rp * (BLK / RP)] != ODMA_SLOT_NONE && row[rp] < a.n_rows;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      cs[rp][e] = 1.f;
      sn[rp][e] = 0.f;
      if (there[rp] && turned && h0 < a.Hq + a.Hkv) {
        const int f = 4 * u + e;
        const double turns = (double)a.positions[(int64_t)a.axis[f] * a.n_rows + row[rp]] * ((double)a.inv_freq[f] * 0.15915494309189535);
        sincospif(2.f * (float)(turns - rint(turns)), &sn[rp][e], &cs[rp][e]);
      }
    }
  }
  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 1.f;
  if (in_head && a.q_weight) {
    load4((const T*)a.q_weight + ca, wq, 0);
    load4((const T*)a.q_weight + cb, wq, 4);
  }
  if (in_head && a.k_weight) {
    load4((const T*)a.k_weight + ca, wk, 0);
    load4((const T*)a.k_weight + cb, wk, 4);
  }
  auto prepare = [&](float (&x)[8], const float (&w)[8], bool norm, int rp) {
    if (norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
#pragma unroll
      for (int o = GROUP / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
      const float inv = 1.f / sqrtf(ss / (float)a.D + a.eps);
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
  // the same heads of all rows of the tile: HB heads from h on, of `src` with `heads` heads
  auto load = [&](float (&x)[NB][RP][8], const T* src, int64_t stride, int h, int end) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int rp = 0; rp < RP; ++rp) {
        const int hh = h + b * HP + sub;
        if (there[rp] && hh < end) {
          const T* p = src + row[rp] * stride + (int64_t)hh * a.D;
          load4(p + ca, x[b][rp], 0);
          load4(p + cb, x[b][rp], 4);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[b][rp][i] = 0.f;
        }
      }
  };

  // ---- queries
  for (int h = h0; h < min(h1, a.Hq); h += HB) {
    float x[NB][RP][8];
    const int end = min(h1, a.Hq);
    load(x, (const T*)a.q, a.q_stride, h, end);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int rp = 0; rp < RP; ++rp) {
        const int hh = h + b * HP + sub;
        prepare(x[b][rp], wq, a.q_weight != nullptr, rp);
        if (there[rp] && hh < end) {
          T* o = (T*)a.q_out + (row[rp] * a.Hq + hh) * a.D;
          store4(o + ca, x[b][rp]);
          store4(o + cb, x[b][rp] + 4);
        }
      }
  }
  // ---- keys, then values: staged, then written piece by piece
  const int64_t block_bytes = (int64_t)BLK * a.D * (int)sizeof(S);
  const int pieces = a.D / X;                              // 16-byte pieces of a head's row
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const int lo = kv ? a.Hkv : 0;                         // heads of this kind: [Hq + lo, Hq + lo + Hkv)
    const int begin = max(h0 - a.Hq - lo, 0), end = min(h1 - a.Hq - lo, a.Hkv);
    for (int h = begin; h < end; h += HB) {
      float x[NB][RP][8];
      if (kv) load(x, (const T*)a.v, a.v_stride, h, end);
      else load(x, (const T*)a.k, a.k_stride, h, end);
      __syncthreads();                                     // the batch before has been written
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int rp = 0; rp < RP; ++rp) {
          if (!kv) prepare(x[b][rp], wk, a.k_weight != nullptr, rp);
          if (FP8)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[b][rp][i] *= kv ? a.v_inv : a.k_inv;
          if (in_head) {
            S* o = stage + ((b * HP + sub) * BLK + row_in + rp * (BLK / RP)) * STRIDE;
            store4(o + ca, x[b][rp]);
            store4(o + cb, x[b][rp] + 4);
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
          // other rows: element by element
          for (unsigned left = singles; left; left &= left - 1) {
            const int t = __builtin_ctz(left);
            const int64_t slot = slots[t];
            S* block = (S*)(plane + slot / BLK * block_bytes);
            for (int d = tid; d < a.D; d += 256)
              block[FP8 ? v_index_fp8((int)(slot % BLK), d) : v_index((int)(slot % BLK), d)] = rows[t * STRIDE + d];
          }
        }
      }
    }
  }
}

}  // namespace
