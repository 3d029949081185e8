// Row-major rows <-> pool block format (append, export) and the migration copy.
#pragma once

#include "block_index.h"
#include "kernels_common.h"

namespace {

// ---------------------------------------------------------------------------------
// append / export: row-major rows <-> pool block format
// ---------------------------------------------------------------------------------
constexpr int APPEND_GRID_X = 512;  // most work-groups per request in a bulk append (each takes every 512th group of 16 rows)
constexpr int APPEND_FILL = 1024;   // work-groups up to which append_kernel deals out the chunks of its rows (beyond, four per
                                    // compute unit, the launch is bound by memory: with 4096, 256 prompts of 100 rows took 10 % more)

// Any storage type of 2 or 4 bytes, any head_dim.  A 16-token group that starts on a block boundary is written block-wise,
// ROW_CHUNK bytes of the rows at a time: a K piece is 16 contiguous source bytes, and goes straight through a register; V
// is staged in LDS, so that a thread writes four tokens of two channels at once (16 or 32 bytes) instead of 2- or 4-byte
// elements all over the block.  Slots past the appended rows keep what they hold.  Bound by memory: the scattered stores
// it replaces cost a partial sector each (164 prompts of 218 138 tokens x 4 heads x 64 in bf16, two layers with migrations
// and export, 1.07 GB: 760 -> 231 us, 4.6 TB/s).  A small launch is bound by round trips instead, which chunks taken in turn
// pile up, so there the third grid dimension deals them out (one prompt of 16 rows of 8 x 256 in fp32: 20.0 us row by row,
// 19.7 in turn, 4.8 dealt out; 64 of 6 rows of 32 x 64 in bf16: 9.7, 12.8, 5.5).  Groups that start inside a block, or hold
// one or two rows (the append of a decode step), go row by row (64 single rows of 8 x 128 in fp32: 3.7 us, 10.0 by the
// block; from three rows on the block wins or is within a microsecond).
constexpr int ROW_CHUNK = 1024;
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(RowArgs a, int32_t n, const int64_t* __restrict__ offsets,
                                                     const int32_t* __restrict__ positions, int32_t pos_bias,
                                                     const int32_t* __restrict__ n_new,
                                                     const int64_t* __restrict__ src_start,
                                                     const int32_t* __restrict__ bt, int32_t bt_stride,
                                                     const T* __restrict__ k_new, const T* __restrict__ v_new) {
  constexpr int X = 16 / sizeof(T);
  constexpr int CE = ROW_CHUNK / sizeof(T), STRIDE = CE + X;         // elements of a chunk, of a staged row (padded)
  constexpr int LOADS = BLK * ROW_CHUNK / 16 / 256;
  __shared__ __attribute__((aligned(16))) T rows[BLK * STRIDE];
  const int r = blockIdx.y;
  const int cnt = n_new ? n_new[r] : 1;
  const int64_t src0 = src_start ? src_start[r] : (int64_t)r;
  const int pos0 = positions[r] + pos_bias;
  if (pos0 < 0) return;
  const int row_elems = a.Hkv * a.D;
  const int chunks = row_elems / X;
  const int64_t block_elems = (int64_t)BLK * a.D;
  // groups of 16 rows are dealt to the work-groups of the request's grid row round-robin: a grid row is at most
  // APPEND_GRID_X wide, however long the longest append of the batch is
  for (int j0 = blockIdx.x * BLK; j0 < cnt; j0 += gridDim.x * BLK) {
    const int have = min(BLK, cnt - j0);
    if ((pos0 + j0) % BLK == 0 && have > 2) {
      const int pos = pos0 + j0;
      const int64_t blk = bt ? (int64_t)bt[(int64_t)r * bt_stride + pos / BLK] : offsets[r] / BLK + pos / BLK;
      for (int e0 = blockIdx.z * CE; e0 < row_elems; e0 += CE * gridDim.z) {   // (a chunk is whole groups of 32 channels)
        const int pieces = min(CE, row_elems - e0) / X;               // 16-byte pieces of a row in this chunk
        uint4v kp[LOADS], vp[LOADS];
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
          const int i = threadIdx.x + 256 * l, t = i & 15, c = i >> 4;
          const bool in = c < pieces && t < have;
          const int64_t src = (src0 + j0 + t) * row_elems + e0 + c * X;
          kp[l] = in ? *(const uint4v*)(k_new + src) : uint4v{0u, 0u, 0u, 0u};
          vp[l] = in ? *(const uint4v*)(v_new + src) : uint4v{0u, 0u, 0u, 0u};
        }
        __syncthreads();                                              // the previous chunk's rows have been read
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
          const int i = threadIdx.x + 256 * l, t = i & 15, c = i >> 4;
          if (c < pieces && t < have) {
            const int e = e0 + c * X, g = e / a.D, d0 = e - g * a.D;
            T* kd = (T*)(a.k + (int64_t)g * a.head_stride) + blk * block_elems;
            *(uint4v*)(kd + k_index(t, d0, X)) = kp[l];
            *(uint4v*)(rows + t * STRIDE + c * X) = vp[l];
          }
        }
        __syncthreads();
        // V: thread -> (32-channel group, token quad, channel c): tokens 4 tq .. +3 of channels c and 16 + c of the group
        for (int i = threadIdx.x; i < pieces * X * 2; i += 256) {     // 64 per group of 32 channels
          const int c = i & 15, tq = (i >> 4) & 3, gr = i >> 6, valid = have - 4 * tq;
          const int e = e0 + gr * 32, g = e / a.D, d0 = e - g * a.D;
          T* vd = (T*)(a.v + (int64_t)g * a.head_stride) + blk * block_elems + v_index(4 * tq, d0 + c);
          alignas(16) T piece[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            piece[k] = rows[(4 * tq + k) * STRIDE + gr * 32 + c];
            piece[4 + k] = rows[(4 * tq + k) * STRIDE + gr * 32 + 16 + c];
          }
          if (valid >= 4) {
#pragma unroll
            for (int k = 0; k < (int)sizeof(piece) / 16; ++k) ((uint4v*)vd)[k] = ((const uint4v*)piece)[k];
          } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
              if (k < valid) {
                vd[k] = piece[k];
                vd[4 + k] = piece[4 + k];
              }
          }
        }
      }
      continue;
    }
    for (int j = j0; j < j0 + have; ++j) {
      const int pos = pos0 + j;
      const int64_t blk = bt ? (int64_t)bt[(int64_t)r * bt_stride + pos / BLK] : offsets[r] / BLK + pos / BLK;
      const int t = pos % BLK;
      const T* ks = k_new + (src0 + j) * row_elems;
      const T* vs = v_new + (src0 + j) * row_elems;
      for (int c = blockIdx.z * blockDim.x + threadIdx.x; c < chunks; c += blockDim.x * gridDim.z) {
        const int e0 = c * X, g = e0 / a.D, d0 = e0 % a.D;
        T* kd = (T*)(a.k + (int64_t)g * a.head_stride) + blk * block_elems;
        T* vd = (T*)(a.v + (int64_t)g * a.head_stride) + blk * block_elems;
        *(uint4v*)(kd + k_index(t, d0, X)) = *(const uint4v*)(ks + e0);
        alignas(16) T tmp[X];
        *(uint4v*)tmp = *(const uint4v*)(vs + e0);
#pragma unroll
        for (int i = 0; i < X; ++i) vd[v_index(t, d0 + i)] = tmp[i];
      }
    }
  }
}

// bf16, head_dim 128: a 16-token group that starts on a block boundary is written block-wise -- K pieces are
// 16 contiguous source bytes anyway; V is staged through LDS so that its pieces (four tokens of two channels)
// leave as whole 16-byte stores instead of sixteen thousand 2-byte ones per block.  Token slots of the block
// past the appended rows get zeros (they lie past the request's length and are rewritten before they are read).
// Groups that do not start on a block boundary (the one-row append of a decode step) take the row-wise path.
__global__ __launch_bounds__(256) void append_bf16_d128_kernel(RowArgs a, int32_t n, const int64_t* __restrict__ offsets,
                                                               const int32_t* __restrict__ positions, int32_t pos_bias,
                                                               const int32_t* __restrict__ n_new,
                                                               const int64_t* __restrict__ src_start,
                                                               const int32_t* __restrict__ bt, int32_t bt_stride,
                                                               const unsigned short* __restrict__ k_new,
                                                               const unsigned short* __restrict__ v_new) {
  __shared__ __attribute__((aligned(16))) unsigned short rows[BLK * 128];
  const int r = blockIdx.y;
  const int cnt = n_new ? n_new[r] : 1;
  const int64_t src0 = src_start ? src_start[r] : (int64_t)r;
  const int pos0 = positions[r] + pos_bias;
  if (pos0 < 0) return;
  const int row_elems = a.Hkv * 128;
  const int64_t block_elems = (int64_t)BLK * 128;
  for (int j0 = blockIdx.x * BLK; j0 < cnt; j0 += gridDim.x * BLK) {   // (the trip count is the same for the whole work-group)
  const int j1 = min(j0 + BLK, cnt);
  if ((pos0 + j0) % BLK == 0) {
    const int pos = pos0 + j0;
    const int64_t blk = bt ? (int64_t)bt[(int64_t)r * bt_stride + pos / BLK] : offsets[r] / BLK + pos / BLK;
    const int p = threadIdx.x;                               // one 16-byte piece of the K block and of the V block
    const int t = p & 15, c8 = p >> 4;                       // K piece: token t, channels 8 c8 .. +7
    const int tq = (p >> 4) & 3, c = p & 15, k32 = p >> 6;   // V piece: tokens 4 tq .. +3 of channels 32 k32 + c and + 16
    for (int g = 0; g < a.Hkv; ++g) {
      const bool have = j0 + t < j1;
      const int64_t src = (src0 + j0 + t) * row_elems + g * 128 + c8 * 8;
      const uint4v zero = {0u, 0u, 0u, 0u};
      const uint4v kp = have ? *(const uint4v*)(k_new + src) : zero;
      const uint4v vp = have ? *(const uint4v*)(v_new + src) : zero;
      unsigned short* kd = (unsigned short*)(a.k + (int64_t)g * a.head_stride) + blk * block_elems;
      *(uint4v*)(kd + p * 8) = kp;                           // k_index(t, 8 c8, 8) = (c8 * 16 + t) * 8 = p * 8
      __syncthreads();                                       // the previous head's pieces have been read
      *(uint4v*)(rows + t * 128 + c8 * 8) = vp;
      __syncthreads();
      alignas(16) unsigned short piece[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        piece[i] = rows[(4 * tq + i) * 128 + 32 * k32 + c];
        piece[4 + i] = rows[(4 * tq + i) * 128 + 32 * k32 + 16 + c];
      }
      unsigned short* vd = (unsigned short*)(a.v + (int64_t)g * a.head_stride) + blk * block_elems;
      *(uint4v*)(vd + p * 8) = *(const uint4v*)piece;        // v_index(4 tq, 32 k32 + c) = ((k32 * 4 + tq) * 16 + c) * 8 = p * 8
    }
    continue;
  }
  const int chunks = row_elems / 8;
  for (int j = j0; j < j1; ++j) {
    const int pos = pos0 + j;
    const int64_t blk = bt ? (int64_t)bt[(int64_t)r * bt_stride + pos / BLK] : offsets[r] / BLK + pos / BLK;
    const int t = pos % BLK;
    const unsigned short* ks = k_new + (src0 + j) * row_elems;
    const unsigned short* vs = v_new + (src0 + j) * row_elems;
    for (int c = threadIdx.x; c < chunks; c += blockDim.x) {
      const int e0 = c * 8, g = e0 >> 7, d0 = e0 & 127;
      unsigned short* kd = (unsigned short*)(a.k + (int64_t)g * a.head_stride) + blk * block_elems;
      unsigned short* vd = (unsigned short*)(a.v + (int64_t)g * a.head_stride) + blk * block_elems;
      *(uint4v*)(kd + k_index(t, d0, 8)) = *(const uint4v*)(ks + e0);
      alignas(16) unsigned short tmp[8];
      *(uint4v*)tmp = *(const uint4v*)(vs + e0);
#pragma unroll
      for (int i = 0; i < 8; ++i) vd[v_index(t, d0 + i)] = tmp[i];
    }
  }
  }
}

// Export: a work-group takes GATHER_CHUNK bytes of the rows of one 16-token group, one K piece and one or two V pieces per
// thread; V pieces are read whole and turned into rows in LDS.  Bound by its round trips (block id, pieces, rows), so every
// chunk has a work-group of its own: with 1 KiB chunks taken in turn by one work-group, a short export of rows of several
// KiB took up to ten times what reading token by token had (16 tokens of 8 heads x 256 in fp32: 3.3 -> 15.6 us, now 2.9; of
// 32 x 128 in bf16: 4.4 -> 18.6, now 2.9; 8000 tokens of 4 x 128 in bf16: 18.3 -> 8.2, now 7.3).
constexpr int GATHER_CHUNK = 256;
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(RowArgs a, int64_t offset, int32_t length,
                                                     const int32_t* __restrict__ block_row,
                                                     T* __restrict__ k_out, T* __restrict__ v_out) {
  constexpr int X = 16 / sizeof(T);
  constexpr int CE = GATHER_CHUNK / sizeof(T), STRIDE = CE + X;
  __shared__ __attribute__((aligned(16))) T rows[BLK * STRIDE];
  const int row_elems = a.Hkv * a.D;
  const int64_t block_elems = (int64_t)BLK * a.D;
  const int e0 = blockIdx.y * CE, pieces = min(CE, row_elems - e0) / X;
  // K: thread -> (piece c, token t); V: thread -> (32-channel group, token quad, channel of its first half)
  const int t = threadIdx.x & 15, c = threadIdx.x >> 4;
  const int ek = e0 + c * X, gk = ek / a.D, dk = ek - gk * a.D;
  const int cv = threadIdx.x & 15, tq = (threadIdx.x >> 4) & 3, gr = threadIdx.x >> 6;
  const int ev = e0 + gr * 32, gv = ev / a.D, dv = ev - gv * a.D;
  const bool has_k = c < pieces, has_v = gr * 32 < pieces * X;
  const T* kd = (const T*)(a.k + (int64_t)gk * a.head_stride) + k_index(t, dk, X);
  const T* vd = (const T*)(a.v + (int64_t)gv * a.head_stride) + v_index(4 * tq, dv + cv);
  for (int64_t p0 = (int64_t)blockIdx.x * BLK; p0 < length; p0 += (int64_t)gridDim.x * BLK) {
    const int have = (int)min((int64_t)BLK, length - p0);
    const int64_t at = (block_row ? (int64_t)block_row[p0 / BLK] : offset / BLK + p0 / BLK) * block_elems;
    uint4v kp = {0u, 0u, 0u, 0u};
    alignas(16) T piece[8];
    if (has_v)
#pragma unroll
      for (int k = 0; k < (int)sizeof(piece) / 16; ++k) ((uint4v*)piece)[k] = ((const uint4v*)(vd + at))[k];
    if (has_k) kp = *(const uint4v*)(kd + at);
    __syncthreads();                                                  // the previous group's rows have left
    if (has_v)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        rows[(4 * tq + k) * STRIDE + gr * 32 + cv] = piece[k];
        rows[(4 * tq + k) * STRIDE + gr * 32 + 16 + cv] = piece[4 + k];
      }
    __syncthreads();
    if (has_k && t < have) {
      const int64_t dst = (p0 + t) * row_elems + ek;
      *(uint4v*)(k_out + dst) = kp;
      *(uint4v*)(v_out + dst) = *(const uint4v*)(rows + t * STRIDE + c * X);
    }
  }
}

// ---------------------------------------------------------------------------------
// fp8 storage (head_dim 128): a block is 16 tokens x 128 bytes, laid out as the operands of the
// 16x16x32 fp8 matrix instruction.  K: lane (t, g4) of a wave reads, for each 64-channel half k, 16 bytes =
// channels 64k + 8 g4 .. +8 and 64k + 32 + 8 g4 .. +8 of token t.  V: lane (c, q) reads, per half k,
// 16 bytes = for each of the four 16-channel groups of the half, channel c of tokens 4q .. 4q+3.
// ---------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void append_fp8_kernel(RowArgs a, int32_t n, const int64_t* __restrict__ offsets,
                                                         const int32_t* __restrict__ positions, int32_t pos_bias,
                                                         const int32_t* __restrict__ n_new,
                                                         const int64_t* __restrict__ src_start,
                                                         const int32_t* __restrict__ bt, int32_t bt_stride,
                                                         const unsigned char* __restrict__ k_new,
                                                         const unsigned char* __restrict__ v_new) {
  const int r = blockIdx.y;
  const int cnt = n_new ? n_new[r] : 1;
  const int64_t src0 = src_start ? src_start[r] : (int64_t)r;
  const int pos0 = positions[r] + pos_bias;
  if (pos0 < 0) return;
  const int row_elems = a.Hkv * 128;
  const int chunks = row_elems / 8;
  const int64_t block_bytes = (int64_t)BLK * 128;
  __shared__ __attribute__((aligned(16))) unsigned char vrows[BLK * 128];
  for (int j0 = blockIdx.x * BLK; j0 < cnt; j0 += gridDim.x * BLK) {   // (the trip count is the same for the whole work-group)
  const int j1 = min(j0 + BLK, cnt);
  if ((pos0 + j0) % BLK == 0) {
    // A 16-token group that starts on a block boundary is written block-wise, as whole 16-byte pieces (token slots
    // past the appended rows get zeros).  A K piece is two 8-byte runs of one source row; a V piece gathers four
    // tokens of four channels, so the V rows of the group go through LDS.
    const int pos = pos0 + j0;
    const int64_t blk = bt ? (int64_t)bt[(int64_t)r * bt_stride + pos / BLK] : offsets[r] / BLK + pos / BLK;
    const int tid = threadIdx.x;
    const int p = tid & 127;                                 // piece of the K block (threads 0..127) or of the V block (128..255)
    const int kt = p & 15, kq = (p >> 4) & 3, kj = p >> 6;   // K piece: token kt, channels 64 kj + 8 kq .. +7 and + 32
    const int vc = p & 15, vq = (p >> 4) & 3, vj = p >> 6;   // V piece: tokens 4 vq .. +3 of channels 64 vj + 16 w + vc, w < 4
    const int st = tid >> 4, sc = tid & 15;                  // staging: 8 bytes of token st
    for (int g = 0; g < a.Hkv; ++g) {
      const uint2v zero = {0u, 0u};
      const uint2v sv = j0 + st < j1 ? *(const uint2v*)(v_new + (src0 + j0 + st) * row_elems + g * 128 + sc * 8) : zero;
      __syncthreads();                                       // the previous head's pieces have been read
      *(uint2v*)(vrows + st * 128 + sc * 8) = sv;
      __syncthreads();
      if (tid < 128) {
        const bool have = j0 + kt < j1;
        const unsigned char* src = k_new + (src0 + j0 + kt) * row_elems + g * 128 + 64 * kj + 8 * kq;
        const uint2v lo = have ? *(const uint2v*)src : zero, hi = have ? *(const uint2v*)(src + 32) : zero;
        unsigned char* kd = (unsigned char*)a.k + (int64_t)g * a.head_stride + blk * block_bytes;
        *(uint4v*)(kd + p * 16) = uint4v{lo[0], lo[1], hi[0], hi[1]};   // k_index_fp8(kt, 64 kj + 8 kq) = p * 16
      } else {
        alignas(16) unsigned char piece[16];
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) piece[4 * w + i] = vrows[(4 * vq + i) * 128 + 64 * vj + 16 * w + vc];
        unsigned char* vd = (unsigned char*)a.v + (int64_t)g * a.head_stride + blk * block_bytes;
        *(uint4v*)(vd + p * 16) = *(const uint4v*)piece;     // v_index_fp8(4 vq, 64 vj + vc) = p * 16
      }
    }
    continue;
  }
  for (int j = j0; j < j1; ++j) {
    const int pos = pos0 + j;
    const int64_t blk = bt ? (int64_t)bt[(int64_t)r * bt_stride + pos / BLK] : offsets[r] / BLK + pos / BLK;
    const int t = pos % BLK;
    const unsigned char* ks = k_new + (src0 + j) * row_elems;
    const unsigned char* vs = v_new + (src0 + j) * row_elems;
    for (int c = threadIdx.x; c < chunks; c += blockDim.x) {
      const int e0 = c * 8, g = e0 >> 7, d0 = e0 & 127;
      unsigned char* kd = (unsigned char*)a.k + (int64_t)g * a.head_stride + blk * block_bytes;
      unsigned char* vd = (unsigned char*)a.v + (int64_t)g * a.head_stride + blk * block_bytes;
      *(uint2v*)(kd + k_index_fp8(t, d0)) = *(const uint2v*)(ks + e0);
      alignas(8) unsigned char tmp[8];
      *(uint2v*)tmp = *(const uint2v*)(vs + e0);
#pragma unroll
      for (int i = 0; i < 8; ++i) vd[v_index_fp8(t, d0 + i)] = tmp[i];
    }
  }
  }
}

__global__ __launch_bounds__(256) void gather_fp8_kernel(RowArgs a, int64_t offset, int32_t length,
                                                         const int32_t* __restrict__ block_row,
                                                         unsigned char* __restrict__ k_out,
                                                         unsigned char* __restrict__ v_out) {
  const int row_elems = a.Hkv * 128;
  const int chunks = row_elems / 8;
  const int64_t block_bytes = (int64_t)BLK * 128;
  for (int pos = blockIdx.x; pos < length; pos += gridDim.x) {
    const int64_t blk = block_row ? (int64_t)block_row[pos / BLK] : offset / BLK + pos / BLK;
    const int t = pos % BLK;
    for (int c = threadIdx.x; c < chunks; c += blockDim.x) {
      const int e0 = c * 8, g = e0 >> 7, d0 = e0 & 127;
      const unsigned char* kd = (const unsigned char*)a.k + (int64_t)g * a.head_stride + blk * block_bytes;
      const unsigned char* vd = (const unsigned char*)a.v + (int64_t)g * a.head_stride + blk * block_bytes;
      *(uint2v*)(k_out + (int64_t)pos * row_elems + e0) = *(const uint2v*)(kd + k_index_fp8(t, d0));
      alignas(8) unsigned char tmp[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) tmp[i] = vd[v_index_fp8(t, d0 + i)];
      *(uint2v*)(v_out + (int64_t)pos * row_elems + e0) = *(uint2v*)tmp;
    }
  }
}

// ---------------------------------------------------------------------------------
// migration copy: for every (layer, KV head, K|V) one linear run of whole blocks
// ---------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void migrate_copy_kernel(char* k_pool, char* v_pool, int64_t plane_stride,
                                                           int64_t src_byte, int64_t dst_byte, int64_t n_bytes) {
  // blockIdx.y = plane (layer * Hkv + head) * 2 + {0: K, 1: V}
  const int plane = blockIdx.y >> 1;
  char* base = ((blockIdx.y & 1) ? v_pool : k_pool) + (int64_t)plane * plane_stride;
  const uint4v* src = (const uint4v*)(base + src_byte);
  uint4v* dst = (uint4v*)(base + dst_byte);
  const int64_t n16 = n_bytes / 16;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += (int64_t)gridDim.x * blockDim.x)
    dst[i] = src[i];
}

// the same for up to MIGRATE_BATCH_MAX requests in one launch: blockIdx.z = request of the batch
constexpr int MIGRATE_BATCH_MAX = 16;
struct MigrateBatch {
  int64_t src_byte[MIGRATE_BATCH_MAX], dst_byte[MIGRATE_BATCH_MAX], n_bytes[MIGRATE_BATCH_MAX];
  int32_t n;
};
__global__ __launch_bounds__(256) void migrate_batch_kernel(char* k_pool, char* v_pool, int64_t plane_stride, MigrateBatch mb) {
  const int plane = blockIdx.y >> 1, q = blockIdx.z;
  char* base = ((blockIdx.y & 1) ? v_pool : k_pool) + (int64_t)plane * plane_stride;
  const uint4v* src = (const uint4v*)(base + mb.src_byte[q]);
  uint4v* dst = (uint4v*)(base + mb.dst_byte[q]);
  const int64_t n16 = mb.n_bytes[q] / 16;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += (int64_t)gridDim.x * blockDim.x)
    dst[i] = src[i];   // ordinary accesses: the streaming hints measured 15 % slower for a copy
}

// ---------------------------------------------------------------------------------
// read probe: every work-group strides through the whole buffer, 8 loads of 16 B per lane in flight
// ---------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void read_probe_kernel(const uint4v* __restrict__ p, size_t n16, unsigned* sink) {
  const size_t stride = (size_t)gridDim.x * blockDim.x;
  size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  unsigned acc = 0;
  for (; i + 7 * stride < n16; i += 8 * stride) {
    uint4v v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = __builtin_nontemporal_load(p + i + u * stride);
#pragma unroll
    for (int u = 0; u < 8; ++u) acc += v[u][0] ^ v[u][1] ^ v[u][2] ^ v[u][3];
  }
  for (; i < n16; i += stride) {
    const uint4v v = __builtin_nontemporal_load(p + i);
    acc += v[0] ^ v[1] ^ v[2] ^ v[3];
  }
  if (acc == 0x12345678u) *sink = acc;
}

// ---------------------------------------------------------------------------------
// block probe: the read pattern of the attention kernel without its arithmetic.  Every wave streams an equal share
// of n_steps steps; a step reads the 4 KiB block table[s] of a "K" plane and of a "V" plane (four 16-byte loads per
// lane and plane, streaming), double buffered, the block id fetched one step ahead through the scalar path.  With
// table = identity the blocks form one contiguous slab; with a permutation they are what a paged pool looks like.
// ---------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void block_probe_kernel(const char* __restrict__ k_plane, const char* __restrict__ v_plane,
                                                          const int32_t* __restrict__ table, int64_t n_steps,
                                                          unsigned* sink) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t n_waves = (int64_t)gridDim.x * 4, w = (int64_t)blockIdx.x * 4 + wv;
  const int64_t per = (n_steps + n_waves - 1) / n_waves;
  const int64_t s0 = w * per, s1 = min(s0 + per, n_steps);
  if (s0 >= s1) return;
  const const_i32* tab = as_constant(table);
  const char* kb = k_plane + lane * 16;
  const char* vb = v_plane + lane * 16;
  unsigned acc = 0;
  uint4v bk[2][4], bv[2][4];
  int64_t blk = tab[s0], blk_next = tab[min(s0 + 1, s1 - 1)];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bk[0][j] = __builtin_nontemporal_load((const uint4v*)(kb + blk * 4096 + j * 1024));
    bv[0][j] = __builtin_nontemporal_load((const uint4v*)(vb + blk * 4096 + j * 1024));
  }
  for (int64_t s = s0; s < s1; s += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      blk = blk_next;
      blk_next = tab[min(s + u + 2, s1 - 1)];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bk[(u + 1) % 2][j] = __builtin_nontemporal_load((const uint4v*)(kb + blk * 4096 + j * 1024));
        bv[(u + 1) % 2][j] = __builtin_nontemporal_load((const uint4v*)(vb + blk * 4096 + j * 1024));
      }
      if (s + u < s1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc += bk[u][j][0] ^ bk[u][j][3] ^ bv[u][j][1] ^ bv[u][j][2];
      }
    }
  }
  if (acc == 0x12345678u) *sink = acc;
}

}  // namespace
