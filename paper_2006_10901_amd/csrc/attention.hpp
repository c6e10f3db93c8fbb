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
// per lane.  Left operands of the second kind come from LDS reads that transpose.  All sums, the scores and their statistics are fp32.
//
// Single precision: fp32 instructions do a sixteenth of the fp16 ones' work in the same time, so a number is two fp16 terms, taken times
// a power of two that brings the largest of its head (all heads of a group) to 2^14 .. 2^15.  Two terms hold a number to 2^-23 of itself, or to
// 2^-39 of the largest if that is more.  Of the four products of terms the smallest, at most 2^-22 of the whole, is left out.
// The terms are made once per call, by two small kernels, rather than by every workgroup that reads them; those of Q in the forward pass,
// which one workgroup reads, by that (8 sequences, 8 heads of 40 on two, 723 x 101: 31.9 -> 18.4 us; 8 heads of 128, 710 x 143: 63 -> 58).
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
  int span, buckets, splits, by_length;
  float scale;
  AttnStrides q, kk, v, o, dout, dq, dk, dv;
  const void *Q, *K, *V, *dO;
  // The operands as fp16 terms, `width` of them per row: the caller's arrays in half precision, else arrays of two terms per number,
  // and what the numbers of the sequence's (kv) heads were multiplied by, four factors for each: Q, K, V, dO
  const _Float16 *q16, *k16, *v16, *g16;
  AttnStrides q16s, k16s, v16s, g16s;
  int width;
  const float* factors;
  const int *lengths, *positions, *bucket_of;
  const void* table;
  const uint64_t* mask;
  void* O;
  float* lse;
  void *dQ, *dK, *dV;
  float* delta;          // workspace, of each row: D, what its weights are taken times, the sums of dS at the bias's ends
  float* weight;
  float* ends;
  float* top;            // and what its P is relative to
  int* large;            // and of each 32 rows of a head, from panel to panel: kLarge, kLargeLse
  float* part;           // workspace: what splits leave for the join
  float2* part_sum;      // and of each row its maximum and its sum relative to that (not lse: beside a maximum of 1e9 the sum would be lost)
  double* row_sums;      // workspace: of every split and row, the sums over its keys
  unsigned* again;       // workspace, with a mask: of each wave of a panel kernel, which of its rows are not finite
  float* part_bias;      // workspace: sums of dS by relative position, one set of 2 span + 1 per panel
  int bias_from, bias_splits;   // from which workgroup of attention_dkv_kernel on they make those sums, and over how many a panel is split
};

// The sparse matrix as bits, in words of 64: for every tile of 64 columns a word per row (row_words), for every tile of 64 rows a word
// per column (col_words), and for every 64 rows (columns) which tiles hold anything (row_tiles, col_tiles).  An eighth of a byte
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

// Weights are taken times 2^14: they are at most 1, and fp16 then holds those down to 2^-28 of the largest with all its bits and down to
// 2^-39 with some (as they are: 2^-14 and 2^-25, and a row of 2^16 even weights would lose most of its bits).
constexpr float kOffset = 14.f;

template <typename T> struct AttnPiece;                  // 16 bytes, and the same at any address of an element
template <> struct AttnPiece<_Float16> {
  typedef f16x8 Type;
  typedef f16x8 Any __attribute__((aligned(2)));
};
template <> struct AttnPiece<float> {
  typedef f32x4 Type;
  typedef f32x4 Any __attribute__((aligned(4)));
};

// 16 bytes of a row of d elements, zeros from d on.
template <typename T>
__device__ __forceinline__ typename AttnPiece<T>::Type attn_load_piece(const T* row, int c0, int d) {
  constexpr int E = 16 / sizeof(T);
  typename AttnPiece<T>::Type v = {};
  if (c0 + E <= d) {
    v = *reinterpret_cast<const typename AttnPiece<T>::Any*>(row + c0);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (c0 + e < d) v[e] = row[c0 + e];
  }
  return v;
}
// The same for rows of whole pieces, without a branch and without looking at what comes (that would wait for it): pieces behind the row's
// end are its last one again.  They meet zeros of the other operand, or columns that are not stored.
template <typename T>
__device__ __forceinline__ typename AttnPiece<T>::Type attn_load_whole_piece(const T* row, int c0, int d) {
  return *reinterpret_cast<const typename AttnPiece<T>::Any*>(row + min(c0, d - 16 / (int)sizeof(T)));
}

// Four neighbouring elements of a row of d, of the parts s, s + step .. that splits left (behind the last one that again): asked for together.
__device__ __forceinline__ void attn_load_parts(f32x4 (&v)[4], const float* part, int splits, int s, int step, int64_t rows, int64_t flat, int c, int d) {
  auto row = [&](int u) { return part + (min(s + u * step, splits - 1) * rows + flat) * d; };
  if (d % 4 == 0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = attn_load_whole_piece<float>(row(u), c, d);
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = attn_load_piece<float>(row(u), c, d);
  }
}

// A tile on its way from memory to LDS, requested a tile ahead into registers, then written: ROWS rows of BYTES bytes, PITCH apart.
template <typename T, int ROWS, int BYTES, int PITCH, int THREADS> struct AttnStage {
  using Piece = typename AttnPiece<T>::Type;
  static constexpr int kElements = 16 / (int)sizeof(T), kPieces = BYTES / 16, kCount = ROWS * kPieces / THREADS;
  static_assert(ROWS * kPieces % THREADS == 0, "whole pieces per thread");
  Piece v[kCount];
  // rows [0, rows) of `base`, `stride` elements apart, of d elements, a multiple of a piece's (rows >= 1); behind them the last one again,
  // whose weights are 0 there.  ROWS rows span less than 2^31 bytes: a whole tile takes one offset per thread and bases that are the
  // workgroup's, no arithmetic of the lanes (with 64-bit products per piece it took a third of their instructions).
  // (Rows of 12 and 24 pieces, which do not divide the threads: an offset per piece.)
  static constexpr bool kEven = THREADS % kPieces == 0;
  struct Offsets { unsigned v[kEven ? 1 : kCount]; };
  static __device__ __forceinline__ Offsets whole_offsets(int64_t stride, int tid) {
    Offsets o;
#pragma unroll
    for (int i = 0; i < (kEven ? 1 : kCount); ++i)
      o.v[i] = (unsigned)((i * THREADS + tid) / kPieces) * (unsigned)(stride * (int)sizeof(T)) + (i * THREADS + tid) % kPieces * 16;
    return o;
  }
  __device__ __forceinline__ void load(const T* base, int64_t stride, int rows, int d, const Offsets& whole, int tid) {
    const char* from = reinterpret_cast<const char*>(base);
    if (rows >= ROWS && d * (int)sizeof(T) == BYTES) {
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        v[i] = *reinterpret_cast<const typename AttnPiece<T>::Any*>(from + (kEven ? i * (THREADS / kPieces) * stride * (int)sizeof(T) : 0) +
                                                                    whole.v[kEven ? 0 : i]);
    } else {
      asm volatile("");
#pragma unroll
      for (int i = 0; i < kCount; ++i) {
        const int at = i * THREADS + tid, row = at / kPieces, c = at % kPieces;
        const unsigned offset = (unsigned)min(row, rows - 1) * (unsigned)(stride * (int)sizeof(T)) + min(c * kElements, d - kElements) * (int)sizeof(T);
        v[i] = *reinterpret_cast<const typename AttnPiece<T>::Any*>(from + offset);
      }
    }
  }
  // the same for any d (one branch around all loads: with one around each, each would be waited for)
  __device__ __forceinline__ void load_block(const T* base, int64_t stride, int rows, int d, int tid) {
    if (d % kElements == 0) {
#pragma unroll
      for (int i = 0; i < kCount; ++i) {
        const int at = i * THREADS + tid, row = at / kPieces, c = at % kPieces * kElements;
        v[i] = attn_load_whole_piece<T>(base + min(row, rows - 1) * stride, c, d);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i) {
        const int at = i * THREADS + tid, row = at / kPieces, c = at % kPieces * kElements;
        v[i] = attn_load_piece<T>(base + min(row, rows - 1) * stride, c, d);
      }
    }
  }
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int at = i * THREADS + tid, row = at / kPieces, c = at % kPieces;
      *reinterpret_cast<Piece*>(lds + row * PITCH + c * 16) = v[i];
    }
  }
};

// Rows of D numbers of TERMS fp16 terms each, the first terms of all, then the second.  In LDS 16 bytes apart from a multiple of the
// banks: lanes that read 16 bytes of 32 rows meet no conflict.  The reads that transpose take 64 bytes of four rows at a time, which then
// meet in fours where a row is a multiple of the banks: in twos if it is 48 bytes apart from it, for which kernels of EACH = 1 workgroup
// to a compute unit have room (128 columns, us: dQ in fp32 114 -> 112, dK and dV 142 -> 138, in fp16 127 -> 122).
template <int D, int TERMS, int EACH = 2> struct AttnTile {
  static constexpr int kBytes = D * TERMS * 2, kPitch = kBytes + (EACH == 1 && kBytes % 256 == 0 ? 48 : 16), kSteps = D / 16;
  // Two tiles (K and V, or Q and dO) at a time, in two sets where two workgroups then fit a compute unit (at 128 columns in fp32 one: their
  // registers let no more in; dK and dV 138 -> 134 us): one is written while the other is read, and the workgroup meets once per tile.
  static constexpr int kPair = 2 * kAttnTile * kPitch, kSets = 2 * kPair <= (D == 128 ? 144 : 72) * 1024 ? 2 : 1;
  // A tile that is only read by the reads that transpose (V in the forward pass), 64 bytes of four rows at a time: an odd multiple of
  // 64 bytes puts those into all 64 banks, where 16 bytes past a multiple of 256 lets four rows meet in one.
  static constexpr int kPitchT = ((kBytes + 63) / 64 | 1) * 64;
  template <int ROWS, int THREADS, int PITCH = kPitch> using Stage = AttnStage<_Float16, ROWS, kBytes, PITCH, THREADS>;
};
// Lanes l and l + 32 together, in both.
__device__ __forceinline__ float attn_max_halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
// The larger of `most` and the finite numbers among four.
__device__ __forceinline__ float attn_largest(float most, const f32x4& v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float m = fabsf(v[e]);
    most = m < __builtin_inff() ? fmaxf(most, m) : most;
  }
  return most;
}
// The power of two that brings the largest of some numbers to 2^14 .. 2^15.
__device__ __forceinline__ int attn_exponent(float most) { return most > 0.f ? min(max(14 - ilogbf(most), -120), 120) : 0; }

// The own operand: pieces of row `lane % 32`, the half of the lane.
template <int D, int TERMS> struct AttnOwn {
  f16x8 v[TERMS][D / 16];
  // base: a row that is there, whether or not this lane's is
  __device__ __forceinline__ void load(const _Float16* base, int64_t offset, bool valid, int d, int half) {
    const _Float16* row = base + (valid ? offset : 0);
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const int c = t * D + (2 * s + half) * 8;
        const f16x8 piece = attn_load_whole_piece<_Float16>(row, c, d);
        v[t][s] = valid && c < d ? piece : f16x8{};
      }
  }
  // The terms of a row of d fp32 numbers, made here; returns what products of them have to be multiplied by, a power of two of the row's.
  __device__ __forceinline__ float load_numbers(const float* base, int64_t offset, bool valid, int d, int half) {
    const float* row = base + (valid ? offset : 0);
    f32x4 x[D / 16][2];
    if (d % 4 == 0) {
#pragma unroll
      for (int s = 0; s < D / 8; ++s) x[s / 2][s % 2] = attn_load_whole_piece<float>(row, (2 * (s / 2) + half) * 8 + 4 * (s % 2), d);
    } else {
#pragma unroll
      for (int s = 0; s < D / 8; ++s) x[s / 2][s % 2] = attn_load_piece<float>(row, (2 * (s / 2) + half) * 8 + 4 * (s % 2), d);
    }
    float most = 0.f;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      if (!valid || (2 * (s / 2) + half) * 8 + 4 * (s % 2) >= d) x[s / 2][s % 2] = f32x4{};
      most = attn_largest(most, x[s / 2][s % 2]);
    }
    const int e = attn_exponent(attn_max_halves(most));
    const float factor = ldexpf(1.f, e);
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float number = x[s][i / 4][i % 4] * factor;
        v[0][s][i] = (_Float16)number;
        v[TERMS - 1][s][i] = (_Float16)(number - (float)v[0][s][i]);
      }
    return ldexpf(1.f, -e);
  }
  __device__ __forceinline__ void negate() {
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int s = 0; s < D / 16; ++s) v[t][s] = -v[t][s];
  }
};

// x += a piece of rows times one of own rows, 16 columns.  In single precision the smallest products first, in the same order whether the rows are
// keys or (QUERIES) queries: a score then has the same bits wherever it is formed.
template <bool QUERIES, int D, int TERMS>
__device__ __forceinline__ void attn_multiply(f32x16& x, const AttnOwn<D, TERMS>& rows, const AttnOwn<D, TERMS>& own, int s) {
  if constexpr (TERMS == 2) {
    constexpr int kFirst = QUERIES ? 0 : 1;
    x = __builtin_amdgcn_mfma_f32_32x32x16_f16(rows.v[kFirst][s], own.v[1 - kFirst][s], x, 0, 0, 0);
    x = __builtin_amdgcn_mfma_f32_32x32x16_f16(rows.v[1 - kFirst][s], own.v[kFirst][s], x, 0, 0, 0);
  }
  x = __builtin_amdgcn_mfma_f32_32x32x16_f16(rows.v[0][s], own.v[0][s], x, 0, 0, 0);
}

// X += (32 rows of the tile) (own)^T
template <int PITCH, bool QUERIES = false, int D, int TERMS>
__device__ __forceinline__ void attn_product(f32x16& x, const char* lds, const AttnOwn<D, TERMS>& own, int lane) {
  const char* row = lds + (lane & 31) * PITCH + (lane >> 5) * 16;
  AttnOwn<D, TERMS> a;
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
#pragma unroll
    for (int t = 0; t < TERMS; ++t) a.v[t][s] = *reinterpret_cast<const f16x8*>(row + t * D * 2 + s * 32);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) attn_multiply<QUERIES>(x, a, own, s);
  // the reads run ahead of the products by four, rather than each product waiting for its own
  constexpr int kReads = TERMS * D / 16, kAhead = kReads < 4 ? kReads : 4, kPer = TERMS == 2 ? 3 : 1;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
  for (int i = kAhead; i < kReads; i += TERMS) {
    __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, TERMS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kPer * kAhead / TERMS, 0);
}

// acc (D x 32, blocks of 32) += (32 rows of the tile)^T X
//
// In half precision X, weights or dS, is rounded to fp16 once, as the matrix instructions take it: an error of the size of that which rounding the
// result costs anyway, and independent of it (2-norm, 8 x 16 heads of 64, 512 x 2048: O 2.8e-4, dQ, dK and dV 2.9e-4 to 3.0e-4, of which rounding the result
// is 2.1e-4).  A second term for what is rounded away would leave 2.1e-4 and takes the forward pass from 50 to 60 us there (128 columns, 4096 x 8192: 311 to
// 422), dQ from 67 to 74, dK and dV from 101 to 116.
template <int PITCH, int D, int TERMS>
__device__ __forceinline__ void attn_product_t(f32x16 (&acc)[D / 32], const char* lds, const f32x16& x, int lane) {
  typedef __attribute__((address_space(3))) s16x4* LdsPtr;
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const int i = lane & 15;
  const char* at = lds + (4 * (lane >> 5) + (i >> 2)) * PITCH + (((lane >> 4) & 1) * 16 + (i & 3) * 4) * 2;
  auto left = [&](int s, int offset) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(at + (16 * s) * PITCH + offset));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(at + (16 * s + 8) * PITCH + offset));
    return __builtin_bit_cast(f16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    f16x8 b, rest;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      b[e] = (_Float16)x[8 * s + e];                     // to nearest: weights cut off would be too small in the mean
      if constexpr (TERMS == 2) rest[e] = (_Float16)(x[8 * s + e] - (float)b[e]);
    }
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) {
      const f16x8 a = left(s, blk * 64);
      if constexpr (TERMS == 2) {
        acc[blk] = __builtin_amdgcn_mfma_f32_32x32x16_f16(left(s, D * 2 + blk * 64), b, acc[blk], 0, 0, 0);
        acc[blk] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, rest, acc[blk], 0, 0, 0);
      }
      acc[blk] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, acc[blk], 0, 0, 0);
    }
  }
}

__device__ __forceinline__ bool attn_finite(float v) { return fabsf(v) < __builtin_inff(); }

__device__ __forceinline__ float attn_sum_halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

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

__device__ __forceinline__ unsigned attn_low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// The bias of one head by relative position, in LDS: entry x is that of relative position x - span - PAD, clamped, so that tiles that
// come near the clamped ends need no clamping of their own: 32 queries and 64 keys (forward) or 32 (backward).
constexpr int kAttnPad = 96, kAttnPadBlock = 64;
__host__ __device__ __forceinline__ int attn_bias_entries(int span, int pad) { return 2 * span + 1 + 2 * pad; }
template <typename T, int PAD>
__device__ __forceinline__ void attn_fill_bias(float* lds, const AttnArgs& a, int head, int tid, int threads) {
  const T* row = static_cast<const T*>(a.table) + (int64_t)head * a.buckets;
  for (int x = tid; x < attn_bias_entries(a.span, PAD); x += threads) {
    const int b = a.bucket_of[min(max(x - PAD, 0), 2 * a.span)];
    lds[x] = (float)row[min(max(b, 0), a.buckets - 1)];
  }
}

// The position of a sequence's first query among its keys; far enough out all positions are the same to a bias.
__device__ __forceinline__ int attn_position(const AttnArgs& a, int batch) {
  return a.positions ? min(max(a.positions[batch], -(1 << 30)), 1 << 30) : 0;
}

template <typename T> constexpr int attn_terms() { return sizeof(T) == 4 ? 2 : 1; }
// How many workgroups of the panel kernels a compute unit holds: those of queries, and those of keys.
template <typename T, int D> constexpr int attn_queries_each() { return D * attn_terms<T>() <= 128 ? 2 : 1; }
template <typename T, int D> constexpr int attn_keys_each() { return D < 128 && D * attn_terms<T>() <= 128 ? 2 : 1; }

// How many of its states a sequence has.
__device__ __forceinline__ int attn_seen(const AttnArgs& a, int batch) { return a.lengths ? min(max(a.lengths[batch], 0), a.k) : a.k; }

// Which sequence and head of K and V a workgroup works for, and which of the `inner` pieces of work that each has.  Runs of neighbouring
// pieces go to one XCD, whose L2 then keeps the K and V (or Q and dO) that they share: workgroup ids are dealt to the eight XCDs in turn.
//
// Sequences of unequal length (by_length: lengths known, at most 64 of them): an XCD still gets whole heads where their number allows, and
// takes the longest sequences first.  Workgroups that start together go to the compute units in turn, 32 of an XCD, and those that meet on
// one share it, so every other 32 are taken from the back: the longest is met by the shortest.  (Eight sequences of a quarter to all of 2048
// states, 16 heads, 512 queries, fp16: 51.7 -> 43.1 us.)
struct AttnPlace {
  int batch, kv_head, piece;
  __device__ __forceinline__ AttnPlace(const AttnArgs& a, int inner) : AttnPlace(a, inner, blockIdx.x, gridDim.x) {}
  __device__ __forceinline__ AttnPlace(const AttnArgs& a, int inner, int id, int total) {
    const int xcd = id & 7;
    if (!a.by_length) {
      const int each = total >> 3, rest = total & 7;
      int work = xcd * each + min(xcd, rest) + (id >> 3);
      piece = work % inner;
      work /= inner;
      batch = work % a.batch;
      kv_head = work / a.batch;
      return;
    }
    const bool own = a.kv_heads % 8 == 0;                 // heads of its own for each XCD
    const int at = own ? id >> 3 : id, all = own ? total >> 3 : total, units = own ? 32 : 256, heads = own ? a.kv_heads >> 3 : a.kv_heads;
    const int turn = at / units, slot = at - turn * units, count = min(units, all - turn * units);
    int work = turn * units + (turn & 1 ? count - 1 - slot : slot);
    piece = work % inner;
    work /= inner;
    kv_head = (own ? xcd * heads : 0) + work % heads;
    const int want = work / heads, lane = threadIdx.x & 63, mine = lane < a.batch ? a.lengths[lane] : INT32_MIN;
    int rank = 0;
    for (int i = 0; i < a.batch; ++i) {
      const int other = __builtin_amdgcn_readlane(mine, i);
      rank += other > mine || (other == mine && i < lane);
    }
    batch = uniform(__builtin_ctzll(__ballot(lane < a.batch && rank == want)));
  }
};

// The panel of 128 queries that a workgroup works on, and which part of the keys.
struct AttnPanelOf {
  int split, panel, batch, kv_head, head, panels;
  __device__ __forceinline__ AttnPanelOf(const AttnArgs& a, int rows) : AttnPanelOf(a, rows, a.splits, blockIdx.x, gridDim.x) {}
  __device__ __forceinline__ AttnPanelOf(const AttnArgs& a, int rows, int splits, int id, int total) {
    panels = (rows + kAttnPanel - 1) / kAttnPanel;
    const AttnPlace at(a, a.group * panels * splits, id, total);
    batch = at.batch, kv_head = at.kv_head;
    split = at.piece % splits;
    const int rest = at.piece / splits;
    panel = rest % panels;
    head = kv_head * a.group + rest / panels;
  }
};
__device__ __forceinline__ void attn_tiles_of_split(const AttnArgs& a, int split, int seen, int& begin, int& end) {
  const int all = (seen + kAttnTile - 1) / kAttnTile;
  begin = (int)((int64_t)all * split / a.splits);
  end = (int)((int64_t)all * (split + 1) / a.splits);
}

// The tiles in which a panel of 128 rows (two sets of 64) sees anything, 64 of them at hand at a time.
struct AttnSeenTiles {
  const uint64_t *a = nullptr, *b = nullptr;
  uint64_t bits = 0;
  int group = -1;
  __device__ __forceinline__ AttnSeenTiles(const uint64_t* mask, int64_t at, int64_t tiles, int64_t sets, int first_row) {
    if (!mask) return;
    const int64_t per = (tiles + 63) / 64;
    a = b = mask + at + (first_row >> 6) * per;
    if ((first_row >> 6) + 1 < sets) b = a + per;
  }
  // the one tile below `end` that the first (or second) 64 rows see, or -1 if they see none or more
  __device__ __forceinline__ int only(bool second, int end) const {
    if (!a) return end == 1 ? 0 : -1;
    int found = -1;
    for (int g = 0; g * 64 < end; ++g) {
      const uint64_t x = (second ? b : a)[g];
      if (!x) continue;
      if (found >= 0 || (x & (x - 1))) return -1;
      found = uniform(g * 64 + (int)__builtin_ctzll(x));
    }
    return found < end ? found : -1;
  }
  // the next one from t on, or `end`
  __device__ __forceinline__ int next(int t, int end) {
    if (!a) return t;
    while (t < end) {
      if (t >> 6 != group) {
        group = t >> 6;
        const uint64_t both = a[group] | b[group];
        bits = (uint64_t)(unsigned)uniform((int)(both >> 32)) << 32 | (unsigned)uniform((int)both);
      }
      const uint64_t left = bits >> (t & 63);
      if (left) return min(end, t + (int)__builtin_ctzll(left));
      t = (t | 63) + 1;
    }
    return end;
  }
};

// Which of a tile's 64 positions a row sees, by the mask, and the first `left` of them.
__device__ __forceinline__ uint64_t attn_word(const uint64_t* words, int row, bool valid) { return words ? valid ? words[row] : 0ull : ~0ull; }
__device__ __forceinline__ uint64_t attn_first(uint64_t word, int left) {
  return left >= 64 ? word : left > 0 ? word & ((1ull << left) - 1) : 0ull;
}

// What products of operands have to be multiplied by: 1 in half precision, whose operands are as they are.
struct AttnFactors { float q, k, v, g; };
template <typename T> __device__ __forceinline__ AttnFactors attn_factors(const AttnArgs& a, int batch, int kv_head) {
  if constexpr (sizeof(T) == 2) return {1.f, 1.f, 1.f, 1.f};
  const float* f = a.factors + ((int64_t)batch * a.kv_heads + kv_head) * 4;
  return {f[0], f[1], f[2], f[3]};
}

// Scores of a block of 32 x 32: the scale and the bias.  from: the entry of the bias table for the lane's column and row 0 of the
// block; a row further on is `STEP` entries further on.
template <int STEP> __device__ __forceinline__ void attn_add_bias(f32x16& x, float scale, const float* from) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, from[STEP * (8 * (r / 4) + r % 4)]);
}
__device__ __forceinline__ void attn_add_constant(f32x16& x, float scale, float bias) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, bias);
}

// One row's running softmax: columns of 32 x 32 scores in 16 registers, two lanes to a column.
struct AttnRunning { float most = -__builtin_inff(), sum = 0.f; };

// How the scores of a tile come from products: s = scale x + bias.  Where one bias goes for all of them (no bias, or a tile at one end of
// it) it takes one instruction per score to be the exponent of a weight, 2^(c x + shift), two numbers that nearly cancel: each is rounded to
// 2^-24 of itself, so that the weight of a score s (without its bias) is off by up to 2.6e-7 |s| of itself.  Where each score has its own bias, or the one
// is so large that scores are lost in it (and have to be, as in any sum of the two), or scores are larger than kAttnLargeScore, they are formed
// first and what they are relative to is subtracted from them: three.  (At 128 the short form costs 3.4e-5 of a weight, a fifteenth of what rounding it
// to fp16 does; at 1e4 it would cost 0.2 %, at 2e7 weights would leave the range of fp16.)
constexpr float kAttnLargeBias = 1e6f, kAttnLargeScore = 128.f;
// Whether the difference of a bias and a row's largest score or lse calls for the long form (not that of a row without weights, whose lse is +inf).
__device__ __forceinline__ bool attn_large(float v) { return fabsf(v) > kAttnLargeScore && attn_finite(v); }
struct AttnScores { float scale; bool formed; float bias; };

// x: NB blocks of products (AttnScores::formed: of scores).  Brings the running maximum up to date, scales what has been summed before,
// and says how a product becomes a weight relative to that maximum: 2^(c x + shift).
struct AttnExponent { float c, shift; };
template <int D, int NB>
__device__ __forceinline__ AttnExponent attn_softmax_step(f32x16 (&x)[NB], AttnRunning& run, f32x16 (&acc)[D / 32], const AttnScores& how) {
  float most = -__builtin_inff();
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, x[b][r]);
  most = attn_max_halves(most);
  if (!how.formed) most = __builtin_fmaf(most, how.scale, how.bias);
  if (__any(most > run.most)) {
    asm volatile("");
    const float now = fmaxf(run.most, most);
    // a column that has seen nothing yet has nothing to be scaled: its factor is 0, and (-inf) - (-inf) is not formed
    const float factor = run.most == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((run.most - now) * kLog2e);
    run.sum *= factor;
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) acc[blk] *= factor;
    run.most = now;
  }
  const float base = run.most == -__builtin_inff() ? 0.f : run.most;
  if (!how.formed) {
    float shift = __builtin_fmaf(how.bias - base, kLog2e, kOffset);
    if (__any(attn_large(how.bias - base))) {
      asm volatile("");
      const float inv = 1.f / how.scale;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[b][r] = (__builtin_fmaf(x[b][r], how.scale, how.bias) - base) * inv;
      shift = kOffset;
    }
    return {how.scale * kLog2e, shift};
  }
  // subtracted first: a bias of the type's lowest value times log2 e would be an infinity
  asm volatile("");
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[b][r] -= base;
  return {kLog2e, kOffset};
}
__device__ __forceinline__ void attn_weights(f32x16& x, AttnRunning& run, const AttnExponent& to) {
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], to.c, to.shift));
    sum += x[r];
  }
  run.sum += sum;
}

// What is multiplied instead of a scale of 0, which would make NaN of the -inf of hidden positions.
constexpr float kAttnLeastScale = 1e-37f;

// v where the bit of register r is set (word: shifted by 4 times the half), else `other`.
__device__ __forceinline__ float attn_select(unsigned word, int r, float v, float other) {
  const int all = __builtin_amdgcn_sbfe((int)word, 8 * (r / 4) + r % 4, 1);
  const int bits = (all & __builtin_bit_cast(int, v)) | (~all & __builtin_bit_cast(int, other));
  return __builtin_bit_cast(float, bits);
}
// Scores that a column does not see become -inf.  word: bit per row of the block.
__device__ __forceinline__ void attn_hide(f32x16& x, unsigned word, int half) {
  asm volatile("");                                      // keeps the caller's branch: two instructions per score are not for every tile
  const unsigned w = word >> (4 * half);
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = attn_select(w, r, x[r], -__builtin_inff());
}

// With a mask, what comes out as Inf or NaN is formed again from the definition, one position at a time: tiles multiply whole rows of V (K,
// Q, dO) by the zeros of positions that a row does not see, and Inf and NaN times 0 are NaN.  A wave has a row (or a key), its lanes
// columns l and l + 64.  The panel kernels leave which of a wave's 32 rows are to be formed again, and a kernel of the same grid looks
// (formed in the panel kernels themselves they cost those 3 to 11 % in registers, whether there was anything to do or not).

// The lanes l and l + 32 whose accumulators are not all finite, as bits of 32 columns.
template <int BLOCKS> __device__ __forceinline__ unsigned attn_not_finite(const f32x16 (&acc)[BLOCKS], bool also) {
  bool bad = also;
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) bad |= !attn_finite(acc[b][r]);
  const uint64_t lanes = __ballot(bad);
  return (unsigned)lanes | (unsigned)(lanes >> 32);
}

struct AttnLane { float a, b; };                          // columns l and l + 64
template <typename T> __device__ __forceinline__ AttnLane attn_lane_row(const T* row, int d, int lane) {
  return {lane < d ? (float)row[lane] : 0.f, lane + 64 < d ? (float)row[lane + 64] : 0.f};
}
__device__ __forceinline__ float attn_lane_dot(const AttnLane& x, const AttnLane& y) {
  float s = __builtin_fmaf(x.a, y.a, x.b * y.b);
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  return s;
}
// Rows of a tensor of the caller's.
template <typename T> __device__ __forceinline__ const T* attn_row(const void* base, const AttnStrides& s, int batch, int head, int64_t row) {
  return static_cast<const T*>(base) + batch * s.batch + head * s.head + row * s.row;
}
// One score; `product`: Q_i . K_j
template <typename T> __device__ __forceinline__ float attn_score(const AttnArgs& a, int batch, int head, int row, int key, float product) {
  float bias = 0.f;
  if (a.table) {
    const int rel = key - row - attn_position(a, batch);
    const int b = a.bucket_of[min(max(rel, -a.span), a.span) + a.span];
    bias = (float)static_cast<const T*>(a.table)[(int64_t)head * a.buckets + min(max(b, 0), a.buckets - 1)];
  }
  return __builtin_fmaf(product, a.scale, bias);
}
// f(key) for every key in [begin, end) that a row sees, or f(row) for every row that sees a key.
template <typename F> __device__ __forceinline__ void attn_each_seen(const uint64_t* words, int64_t stride, int at, int begin, int end, F f) {
  for (int tile = begin / 64; tile * 64 < end; ++tile) {
    uint64_t word = words ? words[(int64_t)tile * stride + at] : ~0ull;
    for (int x = max(begin, tile * 64); x < min(end, tile * 64 + 64); ++x)
      if ((word >> (x & 63)) & 1) f(x);
  }
}

// O over the keys [begin, end) of one row, into `to`; its maximum and its sum relative to that.
template <typename T, typename OUT>
__device__ __forceinline__ float2 attn_exact_forward(const AttnArgs& a, int batch, int head, int row, int begin, int end, OUT* to, int lane) {
  const MaskLayout lay(a.m, a.k);
  const int kv_head = head / a.group;
  const AttnLane q = attn_lane_row(attn_row<T>(a.Q, a.q, batch, head, row), a.d, lane);
  float most = -__builtin_inff(), sum = 0.f;
  AttnLane o = {0.f, 0.f};
  attn_each_seen(a.mask ? a.mask + lay.row_words : nullptr, lay.ti * 64, row, begin, end, [&](int key) {
    if (sum != sum) return;                               // NaN stays NaN
    const AttnLane k = attn_lane_row(attn_row<T>(a.K, a.kk, batch, kv_head, key), a.d, lane);
    const float s = attn_score<T>(a, batch, head, row, key, attn_lane_dot(q, k));
    if (s == -__builtin_inff()) return;
    const AttnLane v = attn_lane_row(attn_row<T>(a.V, a.v, batch, kv_head, key), a.d, lane);
    const float now = fmaxf(most, s), factor = most == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((most - now) * kLog2e);
    const float p = __builtin_amdgcn_exp2f((s - now) * kLog2e);
    most = now;
    sum = __builtin_fmaf(sum, factor, p);
    // (a factor of 0 is for nothing summed, or next to nothing)
    o.a = __builtin_fmaf(p, v.a, factor == 0.f ? 0.f : o.a * factor);
    o.b = __builtin_fmaf(p, v.b, factor == 0.f ? 0.f : o.b * factor);
  });
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum;
  if (lane < a.d) to[lane] = (OUT)(sum != sum ? sum : o.a * inv);
  if (lane + 64 < a.d) to[lane + 64] = (OUT)(sum != sum ? sum : o.b * inv);
  return {most, sum};
}
// The logarithm of a row's sum; that of a row that sees nothing: -inf.
__device__ __forceinline__ float attn_lse(float2 s) { return s.y == 0.f ? -__builtin_inff() : s.x + __builtin_amdgcn_logf(s.y) * kLn2; }

// The weight of a score that lies `above` what it is relative to: by no more than rounding (a score added up in another order), but of 1e9 that is 64 and more.
__device__ __forceinline__ float attn_exact_weight(float above) { return __builtin_amdgcn_exp2f((above > 0.f ? fminf(above, 1.f) : above) * kLog2e); }

// dQ of one row over the keys [begin, end).  weight: what P is taken times.
template <typename T, typename OUT>
__device__ __forceinline__ void attn_exact_dq(const AttnArgs& a, int batch, int head, int row, int begin, int end, float lse, float delta, float weight,
                                              OUT* to, int lane) {
  const MaskLayout lay(a.m, a.k);
  const int kv_head = head / a.group;
  const AttnLane q = attn_lane_row(attn_row<T>(a.Q, a.q, batch, head, row), a.d, lane);
  const AttnLane g = attn_lane_row(attn_row<T>(a.dO, a.dout, batch, head, row), a.d, lane);
  AttnLane out = {0.f, 0.f};
  attn_each_seen(a.mask ? a.mask + lay.row_words : nullptr, lay.ti * 64, row, begin, end, [&](int key) {
    const AttnLane k = attn_lane_row(attn_row<T>(a.K, a.kk, batch, kv_head, key), a.d, lane);
    const float p = weight * attn_exact_weight(attn_score<T>(a, batch, head, row, key, attn_lane_dot(q, k)) - lse);
    const float ds = p * (attn_lane_dot(g, attn_lane_row(attn_row<T>(a.V, a.v, batch, kv_head, key), a.d, lane)) - delta);
    out.a = __builtin_fmaf(ds, k.a, out.a);
    out.b = __builtin_fmaf(ds, k.b, out.b);
  });
  if (lane < a.d) to[lane] = (OUT)(out.a * a.scale);
  if (lane + 64 < a.d) to[lane + 64] = (OUT)(out.b * a.scale);
}

// dK and dV of one key over the tiles [begin, end) of all heads of the group (see attention_dkv_kernel).
template <typename T, typename OUT>
__device__ __forceinline__ void attn_exact_dkv(const AttnArgs& a, int batch, int kv_head, int key, int64_t begin, int64_t end, OUT* dk_to, OUT* dv_to,
                                               int lane) {
  const MaskLayout lay(a.m, a.k);
  const int tiles = (a.m + 63) / 64;
  const AttnLane k = attn_lane_row(attn_row<T>(a.K, a.kk, batch, kv_head, key), a.d, lane);
  const AttnLane v = attn_lane_row(attn_row<T>(a.V, a.v, batch, kv_head, key), a.d, lane);
  AttnLane dk = {0.f, 0.f}, dv = {0.f, 0.f};
  for (int h = 0; h < a.group; ++h) {
    const int head = kv_head * a.group + h;
    const int64_t first = (int64_t)h * tiles, from = begin > first ? begin - first : 0, to = end - first < tiles ? end - first : tiles;
    if (from >= to) continue;
    attn_each_seen(a.mask ? a.mask + lay.col_words : nullptr, lay.tj * 64, key, (int)from * 64, min((int)to * 64, a.m), [&](int row) {
      const int64_t flat = ((int64_t)batch * a.heads + head) * a.m + row;
      const float lse = a.top[flat];
      if (lse == -__builtin_inff()) return;
      const AttnLane q = attn_lane_row(attn_row<T>(a.Q, a.q, batch, head, row), a.d, lane);
      const AttnLane g = attn_lane_row(attn_row<T>(a.dO, a.dout, batch, head, row), a.d, lane);
      const float p = a.weight[flat] * attn_exact_weight(attn_score<T>(a, batch, head, row, key, attn_lane_dot(q, k)) - lse);
      const float ds = p * (attn_lane_dot(g, v) - a.delta[flat]);
      dk.a = __builtin_fmaf(ds, q.a, dk.a), dk.b = __builtin_fmaf(ds, q.b, dk.b);
      dv.a = __builtin_fmaf(p, g.a, dv.a), dv.b = __builtin_fmaf(p, g.b, dv.b);
    });
  }
  if (lane < a.d) dk_to[lane] = (OUT)(dk.a * a.scale), dv_to[lane] = (OUT)dv.a;
  if (lane + 64 < a.d) dk_to[lane + 64] = (OUT)(dk.b * a.scale), dv_to[lane + 64] = (OUT)dv.b;
}

}  // namespace spdl
