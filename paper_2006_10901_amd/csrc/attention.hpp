// Attention in one pass: O = softmax(scale Q K^T + bias) V over the positions that a row sees, and its gradients.
//
// The scores of a tile of keys live in registers only.  All products are tiles of 32 x 32 on the matrix cores, written so that what one
// product leaves is what the next one takes, without a trip through LDS:
//
//   a wave owns 32 columns (queries in the forward pass and for dQ, keys for dK and dV), whose operands stay in its registers, and walks
//   tiles of the other side, which the workgroup keeps in LDS.  X = (tile) (own)^T leaves lane l with column l % 32 and rows
//   8 (r / 4) + 4 (l / 32) + r % 4 in its 16 registers r.  As the right operand of the next product, (tile)^T X, lane l has to hold
//   column l % 32 and any half of the rows, the same half that it takes of the left operand: the order of a sum is free, so the left
//   operand is read from LDS in the order in which the registers hold the right one.
//
// The softmax needs the maximum of a column, which lies in lanes l and l + 32: one exchange per tile.  Statistics of a row are one number
// per lane.  Half precision: products on 32 x 32 x 16 fp16 instructions, left operands of the second kind by LDS reads that transpose.
// Single precision: 32 x 32 x 2 fp32 instructions.  All sums, the scores and their statistics are fp32.
#pragma once
#include "common.hpp"

namespace spdl {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnSpanMax = 1024;      // relative positions that a bias tells apart, each way
constexpr int kAttnBucketsMax = 128;
constexpr int kAttnTile = 64;           // keys (or, for dK and dV, queries) per tile
constexpr int kAttnWaves = 4;
constexpr int kAttnPanel = 32 * kAttnWaves;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttnStrides { int64_t batch, head, row; };

// What a call hands to the kernels.  mask_*: bits of the sparse matrix (see MaskLayout).
struct AttnArgs {
  int batch, heads, kv_heads, group, m, k, d;
  int span, buckets, splits;
  float scale;
  AttnStrides q, kk, v, o, dout, dq, dk, dv;
  const void *Q, *K, *V, *dO;
  const int *lengths, *positions, *bucket_of;
  const void* table;
  const uint64_t* mask;
  void* O;
  float* lse;
  void *dQ, *dK, *dV;
  float* delta;          // workspace, [batch, heads, m]
  float* part;           // workspace: what splits leave for the join
  float* part_lse;
  float* part_bias;      // workspace: sums of dS by relative position, one set of 2 span + 1 per workgroup
};

// The sparse matrix as bits, in words of 64: for every tile of 64 columns a word per row (row_words), for every tile of 64 rows a word
// per column (col_words), and for every 64 rows (columns) which tiles hold anything (row_tiles, col_tiles).  A sixteenth of a byte
// per position each way.
struct MaskLayout {
  int64_t ti, tj, row_words, col_words, row_tiles, col_tiles, words;   // tiles of rows and columns, then offsets in words
  __host__ __device__ MaskLayout(int m, int k) {
    ti = ((int64_t)m + 63) / 64;
    tj = ((int64_t)k + 63) / 64;
    row_words = 0;
    col_words = row_words + tj * ti * 64;
    row_tiles = col_words + ti * tj * 64;
    col_tiles = row_tiles + ti * ((tj + 63) / 64);
    words = col_tiles + tj * ((ti + 63) / 64);
  }
};

template <typename T> struct AttnType;
template <> struct AttnType<_Float16> {
  typedef f16x8 Piece;                                   // 16 bytes
  typedef f16x8 PieceAny __attribute__((aligned(2)));
  // Weights are taken times 2^14: they are at most 1, and fp16 then holds those down to 2^-28 of the largest with all its bits and down
  // to 2^-39 with some (as they are: 2^-14 and 2^-25, and a row of 2^16 even weights would lose most of its bits).
  static constexpr float kOffset = 14.f;
};
template <> struct AttnType<float> {
  typedef f32x4 Piece;
  typedef f32x4 PieceAny __attribute__((aligned(4)));
  static constexpr float kOffset = 0.f;
};

// Rows of D elements in LDS, 16 bytes apart from a multiple of the banks: lanes that read 16 bytes of 32 rows meet no conflict.
template <typename T, int D> struct AttnTile {
  static constexpr int kPiece = 16 / sizeof(T);          // elements per piece
  static constexpr int kPieces = D / kPiece;             // pieces per row
  static constexpr int kPitch = D * (int)sizeof(T) + 16; // bytes per row
  static constexpr int kSteps = D * (int)sizeof(T) / 32; // pieces per row and half of the wave
};

// 16 bytes of a row of d elements, zeros from d on.
template <typename T>
__device__ __forceinline__ typename AttnType<T>::Piece attn_load_piece(const T* row, int c0, int d) {
  using Piece = typename AttnType<T>::Piece;
  constexpr int E = 16 / sizeof(T);
  Piece v = {};
  if (c0 + E <= d) {
    v = *reinterpret_cast<const typename AttnType<T>::PieceAny*>(row + c0);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (c0 + e < d) v[e] = row[c0 + e];
  }
  return v;
}

// A tile on its way from memory to LDS: requested a tile ahead into registers, then written.
template <typename T, int D, int ROWS, int THREADS> struct AttnStage {
  using Tile = AttnTile<T, D>;
  static constexpr int kCount = ROWS * Tile::kPieces / THREADS;
  static_assert(ROWS * Tile::kPieces % THREADS == 0, "whole pieces per thread");
  typename AttnType<T>::Piece v[kCount];
  // rows [0, rows) of `base`, `stride` elements apart; zeros behind them
  __device__ __forceinline__ void load(const T* base, int64_t stride, int rows, int d, int tid) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int at = i * THREADS + tid, row = at / Tile::kPieces, c = at % Tile::kPieces;
      v[i] = typename AttnType<T>::Piece{};
      if (row < rows) v[i] = attn_load_piece<T>(base + (int64_t)row * stride, c * Tile::kPiece, d);
    }
  }
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int at = i * THREADS + tid, row = at / Tile::kPieces, c = at % Tile::kPieces;
      *reinterpret_cast<typename AttnType<T>::Piece*>(lds + row * Tile::kPitch + c * 16) = v[i];
    }
  }
};

template <typename T, int D> using AttnOwn = typename AttnType<T>::Piece[AttnTile<T, D>::kSteps];

// The own operand: pieces of row `lane % 32`, the half of the lane.
template <typename T, int D>
__device__ __forceinline__ void attn_load_own(AttnOwn<T, D>& f, const T* row, bool valid, int d, int half) {
  using Tile = AttnTile<T, D>;
#pragma unroll
  for (int s = 0; s < Tile::kSteps; ++s) {
    f[s] = typename AttnType<T>::Piece{};
    if (valid) f[s] = attn_load_piece<T>(row, (2 * s + half) * Tile::kPiece, d);
  }
}

// X += (32 rows of the tile) (own)^T
template <int D>
__device__ __forceinline__ void attn_product(f32x16& x, const char* lds, const AttnOwn<_Float16, D>& own, int lane) {
  using Tile = AttnTile<_Float16, D>;
  const char* row = lds + (lane & 31) * Tile::kPitch + (lane >> 5) * 16;
#pragma unroll
  for (int s = 0; s < Tile::kSteps; ++s)
    x = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8*>(row + s * 32), own[s], x, 0, 0, 0);
}
template <int D>
__device__ __forceinline__ void attn_product(f32x16& x, const char* lds, const AttnOwn<float, D>& own, int lane) {
  using Tile = AttnTile<float, D>;
  const char* row = lds + (lane & 31) * Tile::kPitch + (lane >> 5) * 16;
#pragma unroll
  for (int s = 0; s < Tile::kSteps; ++s) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(row + s * 32);
#pragma unroll
    for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], own[s][e], x, 0, 0, 0);
  }
}

// acc (D x 32, blocks of 32) += (32 rows of the tile)^T X
template <int D>
__device__ __forceinline__ void attn_product_t(f32x16 (&acc)[D / 32], const char* lds, const f32x16& x, int lane, _Float16) {
  using Tile = AttnTile<_Float16, D>;
  typedef __attribute__((address_space(3))) s16x4* LdsPtr;
  const int i = lane & 15;
  const char* at = lds + (4 * (lane >> 5) + (i >> 2)) * Tile::kPitch + (((lane >> 4) & 1) * 16 + (i & 3) * 4) * 2;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    f16x8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (_Float16)x[8 * s + e];         // to nearest: weights cut off would be too small in the mean
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) {
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(at + (16 * s) * Tile::kPitch + blk * 64));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(at + (16 * s + 8) * Tile::kPitch + blk * 64));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const s16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      acc[blk] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), b, acc[blk], 0, 0, 0);
    }
  }
}
template <int D>
__device__ __forceinline__ void attn_product_t(f32x16 (&acc)[D / 32], const char* lds, const f32x16& x, int lane, float) {
  using Tile = AttnTile<float, D>;
  const char* at = lds + 4 * (lane >> 5) * Tile::kPitch + (lane & 31) * 4;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) {
      const float a = *reinterpret_cast<const float*>(at + (8 * (r / 4) + r % 4) * Tile::kPitch + blk * 128);
      acc[blk] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, x[r], acc[blk], 0, 0, 0);
    }
  }
}

__device__ __forceinline__ float attn_other_half(float v) { return __shfl_xor(v, 32); }

// Stores D x 32 accumulators as rows of the output: lane l has row l % 32, four neighbouring elements at a time.
template <typename T, int D>
__device__ __forceinline__ void attn_store_rows(T* row, bool valid, const f32x16 (&acc)[D / 32], float factor, int d, int half) {
  if (!valid) return;
#pragma unroll
  for (int blk = 0; blk < D / 32; ++blk)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = blk * 32 + g * 8 + half * 4;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = acc[blk][4 * g + e] * factor;
      if (c + 4 <= d) {
        Pack<T, 4>::store(row + c, x);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < d) row[c + e] = (T)x[e];
      }
    }
}

// Which bit of a word belongs to register r of a lane in half h: bit 8 (r / 4) + r % 4 of the word shifted by 4 h.
__device__ __forceinline__ bool attn_bit(unsigned word, int r) { return (word >> (8 * (r / 4) + r % 4)) & 1u; }

__device__ __forceinline__ unsigned attn_low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// The next tile from `t` on (below `end`) in which a set of rows sees anything; `a`, `b`: two sets of bits of tiles (both count), or null.
__device__ __forceinline__ int attn_next_tile(int t, int end, const uint64_t* a, const uint64_t* b) {
  if (!a) return t;
  while (t < end) {
    uint64_t w = a[t >> 6];
    if (b) w |= b[t >> 6];
    w >>= t & 63;
    if (w) return min(end, t + (int)__builtin_ctzll(w));
    t = (t | 63) + 1;
  }
  return end;
}

// The bias of one head by relative position, in LDS: entry x is that of relative position x - span - kAttnPad, clamped, so that a
// pair of tiles that comes near the clamped ends needs no clamping of its own.
constexpr int kAttnPad = 96;
__host__ __device__ __forceinline__ int attn_bias_entries(int span) { return 2 * span + 1 + 2 * kAttnPad; }
template <typename T>
__device__ __forceinline__ void attn_fill_bias(float* lds, const AttnArgs& a, int head, int tid, int threads) {
  const T* row = static_cast<const T*>(a.table) + (int64_t)head * a.buckets;
  for (int x = tid; x < attn_bias_entries(a.span); x += threads) {
    const int b = a.bucket_of[min(max(x - kAttnPad, 0), 2 * a.span)];
    lds[x] = (float)row[min(max(b, 0), a.buckets - 1)];
  }
}

// The position of a sequence's first query among its keys; far enough out all positions are the same to a bias.
__device__ __forceinline__ int attn_position(const AttnArgs& a, int batch) {
  return a.positions ? min(max(a.positions[batch], -(1 << 30)), 1 << 30) : 0;
}

// Runs of neighbouring pieces of work go to one XCD, whose L2 then keeps the K and V (or Q and dO) that they share: workgroup ids are
// dealt to the eight XCDs in turn.
__device__ __forceinline__ int attn_work(int id, int total) {
  const int xcd = id & 7, each = total >> 3, rest = total & 7;
  return xcd * each + min(xcd, rest) + (id >> 3);
}

// One row's running softmax: columns of 32 x 32 scores in 16 registers, two lanes to a column.
struct AttnRunning { float most = -__builtin_inff(), sum = 0.f; };

// x: NB blocks of scores, as the product left them (BIAS: scaled and biased already); turns them into weights relative to the
// running maximum and scales what has been summed before.  c: what the exponent is multiplied by to be one of 2.
template <typename T, int D, int NB, bool BIAS>
__device__ __forceinline__ void attn_softmax_step(f32x16 (&x)[NB], AttnRunning& run, f32x16 (&acc)[D / 32], float c) {
  float most = -__builtin_inff();
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, x[b][r]);
  most = fmaxf(most, attn_other_half(most));
  if (__any(most > run.most)) {
    const float now = fmaxf(run.most, most);
    // a column that has seen nothing yet has nothing to be scaled: its factor is 0, and (-inf) - (-inf) is not formed
    const float factor = run.most == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((run.most - now) * c);
    run.sum *= factor;
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) acc[blk] *= factor;
    run.most = now;
  }
  const float base = run.most == -__builtin_inff() ? 0.f : run.most;
  // Scores of a bias are subtracted first: a bias of the type's lowest value times log2 e would be an infinity.
  const float shift = BIAS ? base : AttnType<T>::kOffset - base * c;
  float sum = 0.f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[b][r] = BIAS ? __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][r] - shift, c, AttnType<T>::kOffset))
                     : __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][r], c, shift));
      sum += x[b][r];
    }
  run.sum += sum;
}

// Scores that a column does not see become -inf.  word: bit per row of the block.
__device__ __forceinline__ void attn_hide(f32x16& x, unsigned word, int half) {
  const unsigned w = word >> (4 * half);
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = attn_bit(w, r) ? x[r] : -__builtin_inff();
}

}  // namespace spdl
