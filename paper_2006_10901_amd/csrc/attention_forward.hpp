// Forward attention: a kernel for panels of 128 queries of a head, one for a few queries (single tokens) that share a head of K and V,
// and the join of what parts of the keys gave.
#pragma once
#include "attention.hpp"

namespace spdl {

// Scores of a block of 32 keys: the scale and the bias.  at: the entry of the bias table for row 0 of the block and the lane's query.
__device__ __forceinline__ void attn_add_bias(f32x16& x, float scale, const float* at) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, at[8 * (r / 4) + r % 4]);
}
__device__ __forceinline__ void attn_add_constant(f32x16& x, float scale, float bias) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, bias);
}

// Panels of 128 queries: a wave has 32 of them, tiles of 64 keys are shared by the four waves.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256) void attention_forward_kernel(const AttnArgs a) {
  using Tile = AttnTile<T, D>;
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  char* lds_k = lds_raw;
  char* lds_v = lds_raw + kAttnTile * Tile::kPitch;
  float* lds_bias = reinterpret_cast<float*>(lds_raw + 2 * kAttnTile * Tile::kPitch);

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  const int panels = (a.m + kAttnPanel - 1) / kAttnPanel;
  int work = attn_work(blockIdx.x, gridDim.x);
  const int split = work % a.splits;
  work /= a.splits;
  const int panel = work % panels;
  work /= panels;
  const int of_group = work % a.group;
  work /= a.group;
  const int batch = work % a.batch, kv_head = work / a.batch, head = kv_head * a.group + of_group;

  const int seen = a.lengths ? min(max(a.lengths[batch], 0), a.k) : a.k;
  const int tiles_all = (a.k + kAttnTile - 1) / kAttnTile;
  const int begin = (int)((int64_t)tiles_all * split / a.splits);
  const int end = min((int)((int64_t)tiles_all * (split + 1) / a.splits), (seen + kAttnTile - 1) / kAttnTile);
  const int first_row = panel * kAttnPanel, wave_row = first_row + wave * 32, row = wave_row + (lane & 31);
  const bool valid = row < a.m;

  const T* Q = static_cast<const T*>(a.Q) + batch * a.q.batch + head * a.q.head;
  const T* K = static_cast<const T*>(a.K) + batch * a.kk.batch + kv_head * a.kk.head;
  const T* V = static_cast<const T*>(a.V) + batch * a.v.batch + kv_head * a.v.head;

  AttnOwn<T, D> q;
  attn_load_own<T, D>(q, Q + (int64_t)row * a.q.row, valid, a.d, half);
  if (a.scale < 0.f) {                                   // so that the largest score is the largest product
#pragma unroll
    for (int s = 0; s < Tile::kSteps; ++s) q[s] = -q[s];
  }
  const float scale = fabsf(a.scale);
  const float c = BIAS ? kLog2e : fmaxf(scale * kLog2e, 1e-37f);   // never 0: it meets the -inf of hidden positions

  const MaskLayout lay(a.m, a.k);
  const uint64_t *tiles_a = nullptr, *tiles_b = nullptr;
  if (a.mask) {
    const int64_t per = (lay.tj + 63) / 64;
    tiles_a = a.mask + lay.row_tiles + (int64_t)(first_row >> 6) * per;
    if ((first_row >> 6) + 1 < lay.ti) tiles_b = tiles_a + per;
  }
  int position = 0;
  if (BIAS) {
    attn_fill_bias<T>(lds_bias, a, head, tid, 256);
    position = attn_position(a, batch);
  }

  f32x16 acc[D / 32] = {};
  AttnRunning run;
  AttnStage<T, D, kAttnTile, 256> stage_k, stage_v;
  int t = attn_next_tile(begin, end, tiles_a, tiles_b);
  if (t < end) {
    stage_k.load(K + (int64_t)t * kAttnTile * a.kk.row, a.kk.row, seen - t * kAttnTile, a.d, tid);
    stage_v.load(V + (int64_t)t * kAttnTile * a.v.row, a.v.row, seen - t * kAttnTile, a.d, tid);
  }
  while (t < end) {
    __syncthreads();
    stage_k.store(lds_k, tid);
    stage_v.store(lds_v, tid);
    __syncthreads();
    const int here = t;
    t = attn_next_tile(t + 1, end, tiles_a, tiles_b);
    if (t < end) {
      stage_k.load(K + (int64_t)t * kAttnTile * a.kk.row, a.kk.row, seen - t * kAttnTile, a.d, tid);
      stage_v.load(V + (int64_t)t * kAttnTile * a.v.row, a.v.row, seen - t * kAttnTile, a.d, tid);
    }
    const int key0 = here * kAttnTile;
    uint64_t word = ~0ull;
    if (a.mask) word = valid ? a.mask[lay.row_words + (int64_t)here * lay.ti * 64 + row] : 0ull;
    if (seen - key0 < 64) word &= (1ull << (seen - key0)) - 1;
    if (wave_row >= a.m || !__any(word != 0)) continue;   // none of the wave's queries sees the tile
    f32x16 x[2] = {};
#pragma unroll
    for (int b = 0; b < 2; ++b) attn_product<D>(x[b], lds_k + b * 32 * Tile::kPitch, q, lane);
    if (BIAS) {
      const int near = key0 - (position + wave_row);     // relative position of the tile's first key and the wave's first query
      if (near - 31 >= a.span || near + 63 <= -a.span) {
        const float far = lds_bias[near > 0 ? 2 * a.span + kAttnPad : kAttnPad];
#pragma unroll
        for (int b = 0; b < 2; ++b) attn_add_constant(x[b], scale, far);
      } else {
        const float* at = lds_bias + kAttnPad + a.span + near - (lane & 31) + 4 * half;
#pragma unroll
        for (int b = 0; b < 2; ++b) attn_add_bias(x[b], scale, at + 32 * b);
      }
    }
    if (__any(word != ~0ull)) {
      attn_hide(x[0], (unsigned)word, half);
      attn_hide(x[1], (unsigned)(word >> 32), half);
    }
    attn_softmax_step<T, D, 2, BIAS>(x, run, acc, c);
#pragma unroll
    for (int b = 0; b < 2; ++b) attn_product_t<D>(acc, lds_v + b * 32 * Tile::kPitch, x[b], lane, T{});
  }

  const float total = run.sum + attn_other_half(run.sum);
  const bool none = run.most == -__builtin_inff() && total == 0.f;
  const float lse = none ? -__builtin_inff() : run.most * c * kLn2 + (__builtin_amdgcn_logf(total) - AttnType<T>::kOffset) * kLn2;
  const float inv = none ? 0.f : 1.f / total;
  const int64_t flat = ((int64_t)batch * a.heads + head) * a.m + row;
  if (a.splits == 1) {
    T* O = static_cast<T*>(a.O) + batch * a.o.batch + head * a.o.head + (int64_t)row * a.o.row;
    attn_store_rows<T, D>(O, valid, acc, inv, a.d, half);
    if (valid && half == 0 && a.lse) a.lse[flat] = lse;
  } else {
    const int64_t rows = (int64_t)a.batch * a.heads * a.m;
    attn_store_rows<float, D>(a.part + (split * rows + flat) * a.d, valid, acc, inv, a.d, half);
    if (valid && half == 0) a.part_lse[split * rows + flat] = lse;
  }
}

// A few queries: the rows of a head of K and V are those of all query heads that share it, m of each, 32 to a workgroup.  K and V are
// read once per 32 rows.  The four waves take blocks of 32 keys in turn, each with its own statistics, and no wave waits for another
// before the end.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256) void attention_token_kernel(const AttnArgs a) {
  using Tile = AttnTile<T, D>;
  constexpr int kBlock = 32 * Tile::kPitch;              // 32 keys or values of a wave
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  char* lds_k = lds_raw + wave * 2 * kBlock;
  char* lds_v = lds_k + kBlock;
  // the bias table of the group's heads, and the bucket of each relative position
  float* lds_table = reinterpret_cast<float*>(lds_raw + kAttnWaves * 2 * kBlock);
  int* lds_bucket = reinterpret_cast<int*>(lds_table + min(a.group, 32) * a.buckets);

  const int rows = a.group * a.m, panels = (rows + 31) / 32;
  int work = blockIdx.x;
  const int split = work % a.splits;
  work /= a.splits;
  const int panel = work % panels;
  work /= panels;
  const int kv_head = work % a.kv_heads, batch = work / a.kv_heads;

  const int seen = a.lengths ? min(max(a.lengths[batch], 0), a.k) : a.k;
  const int blocks_all = (a.k + 31) / 32;
  const int begin = (int)((int64_t)blocks_all * split / a.splits);
  const int end = min((int)((int64_t)blocks_all * (split + 1) / a.splits), (seen + 31) / 32);
  const int packed = panel * 32 + (lane & 31);
  const bool valid = packed < rows;
  const int of_group = valid ? packed / a.m : 0, row = valid ? packed - of_group * a.m : 0;
  const int head = kv_head * a.group + of_group;

  const T* Q = static_cast<const T*>(a.Q) + batch * a.q.batch + head * a.q.head + (int64_t)row * a.q.row;
  const T* K = static_cast<const T*>(a.K) + batch * a.kk.batch + kv_head * a.kk.head;
  const T* V = static_cast<const T*>(a.V) + batch * a.v.batch + kv_head * a.v.head;

  f32x16 acc[D / 32] = {};
  AttnRunning run;
  AttnStage<T, D, 32, 64> stage_k, stage_v;
  int t = begin + wave;
  if (t < end) {
    stage_k.load(K + (int64_t)t * 32 * a.kk.row, a.kk.row, seen - t * 32, a.d, lane);
    stage_v.load(V + (int64_t)t * 32 * a.v.row, a.v.row, seen - t * 32, a.d, lane);
  }
  AttnOwn<T, D> q;
  attn_load_own<T, D>(q, Q, valid, a.d, half);
  if (a.scale < 0.f) {
#pragma unroll
    for (int s = 0; s < Tile::kSteps; ++s) q[s] = -q[s];
  }
  const float scale = fabsf(a.scale);
  const float c = BIAS ? kLog2e : fmaxf(scale * kLog2e, 1e-37f);
  const MaskLayout lay(a.m, a.k);
  int position = 0;
  const float* table = nullptr;
  if (BIAS) {
    const int head0 = panel * 32 / a.m;                  // of the group, the first one in this panel
    const int heads = min(a.group - head0, 32);
    const T* from = static_cast<const T*>(a.table) + (int64_t)(kv_head * a.group + head0) * a.buckets;
    for (int x = tid; x < heads * a.buckets; x += 256) lds_table[x] = (float)from[x];
    for (int x = tid; x < 2 * a.span + 1; x += 256) lds_bucket[x] = min(max(a.bucket_of[x], 0), a.buckets - 1);
    table = lds_table + (valid ? of_group - head0 : 0) * a.buckets;
    position = attn_position(a, batch) + row;
    __syncthreads();
  }
  while (t < end) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    stage_k.store(lds_k, lane);
    stage_v.store(lds_v, lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int key0 = t * 32;
    t += kAttnWaves;
    if (t < end) {
      stage_k.load(K + (int64_t)t * 32 * a.kk.row, a.kk.row, seen - t * 32, a.d, lane);
      stage_v.load(V + (int64_t)t * 32 * a.v.row, a.v.row, seen - t * 32, a.d, lane);
    }
    unsigned word = ~0u;
    if (a.mask) word = valid ? (unsigned)(a.mask[lay.row_words + (int64_t)(key0 >> 6) * lay.ti * 64 + row] >> (key0 & 32)) : 0u;
    word &= attn_low_bits(seen - key0);
    if (!__any(word != 0)) continue;
    f32x16 x[1] = {};
    attn_product<D>(x[0], lds_k, q, lane);
    if (BIAS) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int rel = key0 + 8 * (r / 4) + 4 * half + r % 4 - position;
        x[0][r] = __builtin_fmaf(x[0][r], scale, table[lds_bucket[min(max(rel, -a.span), a.span) + a.span]]);
      }
    }
    if (__any(word != ~0u)) attn_hide(x[0], word, half);
    attn_softmax_step<T, D, 1, BIAS>(x, run, acc, c);
    attn_product_t<D>(acc, lds_v, x[0], lane, T{});
  }

  // the four waves' parts: each scaled to the common maximum, then added up in the waves' order
  __syncthreads();
  float* lds_acc = reinterpret_cast<float*>(lds_raw);                     // [4][32][D + 1]
  float* lds_stat = lds_acc + kAttnWaves * 32 * (D + 1);                  // [4][32][2]
  const float sum = run.sum + attn_other_half(run.sum);
#pragma unroll
  for (int blk = 0; blk < D / 32; ++blk)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      lds_acc[(wave * 32 + (lane & 31)) * (D + 1) + blk * 32 + 8 * (r / 4) + 4 * half + r % 4] = acc[blk][r];
  if (half == 0) {
    lds_stat[(wave * 32 + lane) * 2] = run.most;
    lds_stat[(wave * 32 + lane) * 2 + 1] = sum;
  }
  __syncthreads();
  const int64_t all = (int64_t)a.batch * a.heads * a.m;
  for (int at = tid; at < 32 * a.d; at += 256) {
    const int r = at / a.d, col = at - r * a.d, p = panel * 32 + r;
    if (p >= rows) break;
    const int g = p / a.m, i = p - g * a.m, h = kv_head * a.group + g;
    float most = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) most = fmaxf(most, lds_stat[(w * 32 + r) * 2]);
    float total = 0.f, value = 0.f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      const float own = lds_stat[(w * 32 + r) * 2];
      const float f = own == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((own - most) * c);
      const float s = lds_stat[(w * 32 + r) * 2 + 1], v = lds_acc[(w * 32 + r) * (D + 1) + col];
      // a wave that has seen only NaN has no maximum, and its sums count
      total += s == s ? s * f : s;
      value += v == v ? v * f : v;
    }
    const bool none = most == -__builtin_inff() && total == 0.f;
    const float lse = none ? -__builtin_inff() : most * c * kLn2 + (__builtin_amdgcn_logf(total) - AttnType<T>::kOffset) * kLn2;
    const float result = none ? 0.f : value / total;
    const int64_t flat = ((int64_t)batch * a.heads + h) * a.m + i;
    if (a.splits == 1) {
      (static_cast<T*>(a.O) + batch * a.o.batch + h * a.o.head + (int64_t)i * a.o.row)[col] = (T)result;
      if (col == 0 && a.lse) a.lse[flat] = lse;
    } else {
      a.part[(split * all + flat) * a.d + col] = result;
      if (col == 0) a.part_lse[split * all + flat] = lse;
    }
  }
}

// Joins what the parts of the keys gave: O = sum of exp(lse_s - lse) O_s, in the parts' order.  A wave per row.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnArgs a) {
  const int64_t rows = (int64_t)a.batch * a.heads * a.m;
  const int64_t flat = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (flat >= rows) return;
  const int lane = threadIdx.x & 63;
  float most = -__builtin_inff();
  bool nan = false;
  for (int s = 0; s < a.splits; ++s) {
    const float l = a.part_lse[s * rows + flat];
    nan |= l != l;
    most = fmaxf(most, l);
  }
  float total = 0.f;
  for (int s = 0; s < a.splits && most != -__builtin_inff(); ++s) total += __builtin_amdgcn_exp2f((a.part_lse[s * rows + flat] - most) * kLog2e);
  const float lse = nan ? __builtin_nanf("") : most == -__builtin_inff() ? most : most + __builtin_amdgcn_logf(total) * kLn2;
  const int i = (int)(flat % a.m);
  const int64_t bh = flat / a.m;
  const int h = (int)(bh % a.heads);
  T* O = static_cast<T*>(a.O) + bh / a.heads * a.o.batch + h * a.o.head + (int64_t)i * a.o.row;
  for (int col = lane; col < a.d; col += 64) {
    float value = 0.f;
    for (int s = 0; s < a.splits; ++s) {
      const float l = a.part_lse[s * rows + flat];
      if (l != -__builtin_inff()) value = __builtin_fmaf(__builtin_amdgcn_exp2f((l - lse) * kLog2e), a.part[(s * rows + flat) * a.d + col], value);
    }
    O[col] = (T)value;
  }
  if (lane == 0 && a.lse) a.lse[flat] = lse;
}

// Bits of the sparse matrix, from its CSR topology: cleared, then set by one wave per row.  Which of the threads sets a bit first
// changes nothing.  Column indices out of range are passed over.
__global__ __launch_bounds__(256) void attention_mask_clear_kernel(int64_t words, uint64_t* mask) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < words) mask[i] = 0;
}
__global__ __launch_bounds__(256) void attention_mask_kernel(int m, int k, const int* __restrict__ row_offsets,
                                                             const int* __restrict__ column_indices, unsigned long long* mask) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= m) return;
  const MaskLayout lay(m, k);
  const int64_t per_row = (lay.tj + 63) / 64, per_col = (lay.ti + 63) / 64;
  for (int p = row_offsets[row] + lane; p < row_offsets[row + 1]; p += kWave) {
    const int col = column_indices[p];
    if (col < 0 || col >= k) continue;
    atomicOr(mask + lay.row_words + (int64_t)(col >> 6) * lay.ti * 64 + row, 1ull << (col & 63));
    atomicOr(mask + lay.col_words + (int64_t)(row >> 6) * lay.tj * 64 + col, 1ull << (row & 63));
    atomicOr(mask + lay.row_tiles + (int64_t)(row >> 6) * per_row + (col >> 12), 1ull << ((col >> 6) & 63));
    atomicOr(mask + lay.col_tiles + (int64_t)(col >> 6) * per_col + (row >> 12), 1ull << ((row >> 6) & 63));
  }
}

}  // namespace spdl
