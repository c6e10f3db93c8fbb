// Forward attention: a kernel for panels of 128 queries of a head, one for a few queries (single tokens) that share a head of K and V,
// and the join of what parts of the keys gave.
#pragma once
#include "attention.hpp"

namespace spdl {

// Panels of 128 queries: a wave has 32 of them, tiles of 64 keys are shared by the four waves.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256, (attn_queries_each<T, D>())) void attention_forward_kernel(const AttnArgs a) {
  constexpr int kTerms = attn_terms<T>();
  using Tile = AttnTile<D, kTerms, attn_queries_each<T, D>()>;
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  constexpr int kPair = kAttnTile * (Tile::kPitch + Tile::kPitchT);
  float* lds_bias = reinterpret_cast<float*>(lds_raw + Tile::kSets * kPair);

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  const AttnPanelOf at(a, a.m);
  const int batch = at.batch, head = at.head, kv_head = at.kv_head;
  const int seen = attn_seen(a, batch);
  int begin, end;
  attn_tiles_of_split(a, at.split, seen, begin, end);
  const int first_row = at.panel * kAttnPanel, wave_row = first_row + wave * 32, row = wave_row + (lane & 31);
  const bool valid = row < a.m;

  const _Float16* K = a.k16 + batch * a.k16s.batch + kv_head * a.k16s.head;
  const _Float16* V = a.v16 + batch * a.v16s.batch + kv_head * a.v16s.head;
  const AttnFactors f = attn_factors<T>(a, batch, kv_head);
  AttnOwn<D, kTerms> q;
  float to_score = f.k;
  if constexpr (kTerms == 2)
    to_score *= q.load_numbers(static_cast<const float*>(a.Q) + batch * a.q.batch + head * a.q.head, row * a.q.row, valid, a.d, half);
  else
    q.load(a.q16 + batch * a.q16s.batch + head * a.q16s.head, row * a.q16s.row, valid, a.width, half);
  if (a.scale < 0.f) q.negate();                         // so that the largest score is the largest product
  const float scale = fmaxf(fabsf(a.scale) * to_score, kAttnLeastScale);

  const MaskLayout lay(a.m, a.k);
  AttnSeenTiles tiles(a.mask, lay.row_tiles, lay.tj, lay.ti, first_row);
  int position = 0;
  if (BIAS) {
    attn_fill_bias<T, kAttnPad>(lds_bias, a, head, tid, 256);
    position = attn_position(a, batch);
  }

  f32x16 acc[D / 32] = {};
  AttnRunning run;
  typename Tile::template Stage<kAttnTile, 256> stage_k;
  typename Tile::template Stage<kAttnTile, 256, Tile::kPitchT> stage_v;
  const auto whole_k = stage_k.whole_offsets(a.k16s.row, tid);
  const auto whole_v = stage_v.whole_offsets(a.v16s.row, tid);
  uint64_t word_next = 0;
  auto load = [&](int t) {
    word_next = attn_word(a.mask ? a.mask + lay.row_words + (int64_t)t * lay.ti * 64 : nullptr, row, valid);
    stage_k.load(K + (int64_t)t * kAttnTile * a.k16s.row, a.k16s.row, seen - t * kAttnTile, a.width, whole_k, tid);
    stage_v.load(V + (int64_t)t * kAttnTile * a.v16s.row, a.v16s.row, seen - t * kAttnTile, a.width, whole_v, tid);
  };
  int t = tiles.next(begin, end);
  if (t < end) load(t);
  for (int set = 0; t < end; set ^= Tile::kSets - 1) {
    char* lds_k = lds_raw + set * kPair;
    char* lds_v = lds_k + kAttnTile * Tile::kPitch;
    if (Tile::kSets == 1) __syncthreads();
    stage_k.store(lds_k, tid);
    stage_v.store(lds_v, tid);
    const int key0 = t * kAttnTile;
    const uint64_t word = attn_first(word_next, seen - key0);
    __syncthreads();
    t = tiles.next(t + 1, end);
    if (t < end) load(t);
    if (wave_row >= a.m || !__any(word != 0)) continue;   // none of the wave's queries sees the tile
    f32x16 x[2] = {};
#pragma unroll
    for (int b = 0; b < 2; ++b) attn_product<Tile::kPitch>(x[b], lds_k + b * 32 * Tile::kPitch, q, lane);
    AttnScores how = {scale, false, 0.f};
    if (BIAS) {
      const int near = key0 - (position + wave_row);     // relative position of the tile's first key and the wave's first query
      if (near - 31 >= a.span || near + 63 <= -a.span) {
        how.bias = lds_bias[near > 0 ? 2 * a.span + kAttnPad : kAttnPad];
        how.formed = !(fabsf(how.bias) < kAttnLargeBias);
        if (how.formed) {
#pragma unroll
          for (int b = 0; b < 2; ++b) attn_add_constant(x[b], scale, how.bias);
        }
      } else {
        const float* from = lds_bias + kAttnPad + a.span + near - (lane & 31) + 4 * half;
        how.formed = true;
#pragma unroll
        for (int b = 0; b < 2; ++b) attn_add_bias<1>(x[b], scale, from + 32 * b);
      }
    }
    if (__any(word != ~0ull)) {
      attn_hide(x[0], (unsigned)word, half);
      attn_hide(x[1], (unsigned)(word >> 32), half);
    }
    const AttnExponent to = attn_softmax_step<D, 2>(x, run, acc, how);
    // a wave that has weights to form and multiply goes before one that only multiplies: the vector and the matrix instructions of two
    // waves then meet more often (cross attention of 4096 x 8192, heads of 128: 342 -> 317 us)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      attn_weights(x[b], run, to);
      attn_product_t<Tile::kPitchT, D, kTerms>(acc, lds_v + b * 32 * Tile::kPitchT, x[b], lane);
    }
    __builtin_amdgcn_s_setprio(0);
  }

  const float total = attn_sum_halves(run.sum);
  const bool none = total == 0.f;                        // (NaN is no such sum); weights of 0 times Inf are NaN
  if (none) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b) acc[b] = f32x16{};
  }
  const float2 sum = {run.most, total * __builtin_amdgcn_exp2f(-kOffset)};
  const float inv = none ? 0.f : f.v / total;
  if (a.mask) {
    const unsigned bad = attn_not_finite(acc, !attn_finite(total)) & (unsigned)__ballot(valid);
    if (lane == 0) a.again[blockIdx.x * kAttnWaves + wave] = bad;
  }
  const int64_t flat = ((int64_t)batch * a.heads + head) * a.m + row;
  if (a.splits == 1) {
    T* O = static_cast<T*>(a.O) + batch * a.o.batch + head * a.o.head + (int64_t)row * a.o.row;
    attn_store_rows<T, D>(O, valid, acc, inv, a.d, half);
    if (valid && half == 0 && a.lse) a.lse[flat] = attn_lse(sum);
  } else {
    const int64_t rows = (int64_t)a.batch * a.heads * a.m;
    attn_store_rows<float, D>(a.part + (at.split * rows + flat) * a.d, valid, acc, inv, a.d, half);
    if (valid && half == 0) a.part_sum[at.split * rows + flat] = sum;
  }
}
template <typename T>
__global__ __launch_bounds__(256) void attention_forward_again_kernel(const AttnArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  unsigned left = uniform(a.again[blockIdx.x * kAttnWaves + wave]);
  if (!left) return;
  const AttnPanelOf at(a, a.m);
  int begin, end;
  const int seen = attn_seen(a, at.batch);
  attn_tiles_of_split(a, at.split, seen, begin, end);
  const int64_t flat0 = ((int64_t)at.batch * a.heads + at.head) * a.m, part0 = (int64_t)at.split * a.batch * a.heads * a.m + flat0;
  for (; left; left &= left - 1) {
    const int row = at.panel * kAttnPanel + wave * 32 + __builtin_ctz(left);
    const int last = min(end * kAttnTile, seen);
    if (a.splits == 1) {
      const float2 sum = attn_exact_forward<T>(a, at.batch, at.head, row, begin * kAttnTile, last,
                                               static_cast<T*>(a.O) + at.batch * a.o.batch + at.head * a.o.head + (int64_t)row * a.o.row, lane);
      if (lane == 0 && a.lse) a.lse[flat0 + row] = attn_lse(sum);
    } else {
      const float2 sum = attn_exact_forward<T>(a, at.batch, at.head, row, begin * kAttnTile, last, a.part + (part0 + row) * a.d, lane);
      if (lane == 0) a.part_sum[part0 + row] = sum;
    }
  }
}

// Rows of a head of K and V in the kernels for a few queries: those of all query heads that share it, m of each, ROWS to a workgroup.
template <int ROWS> struct TokenPanel {
  int rows, split, panel, batch, kv_head;
  __device__ __forceinline__ TokenPanel(const AttnArgs& a) {
    rows = a.group * a.m;
    const int panels = (rows + ROWS - 1) / ROWS;
    const AttnPlace at(a, panels * a.splits);
    split = at.piece % a.splits;
    panel = at.piece / a.splits;
    kv_head = at.kv_head;
    batch = at.batch;
  }
};

// Joins PARTS parts of the keys that lie in LDS, each with its own maximum and sum: each is scaled to the common maximum, then they are
// added up in their order.  offset: the power of two that weights were taken times.
template <typename T, int ROWS, int PARTS, int PITCH>
__device__ __forceinline__ void token_finish(const AttnArgs& a, const TokenPanel<ROWS>& at, const float* parts, const float* stats, float offset, int begin,
                                             int end, int tid) {
  __shared__ unsigned bad;                               // with a mask: rows with a result that is not finite
  if (a.mask) {
    if (tid == 0) bad = 0;
    __syncthreads();
  }
  const int64_t all = (int64_t)a.batch * a.heads * a.m;
  for (int x = tid; x < ROWS * a.d; x += 256) {
    const int r = x / a.d, col = x - r * a.d, p = at.panel * ROWS + r;
    if (p >= at.rows) break;
    const int g = p / a.m, i = p - g * a.m, h = at.kv_head * a.group + g;
    float most = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < PARTS; ++w) most = fmaxf(most, stats[(w * ROWS + r) * 2]);
    float total = 0.f, value = 0.f;
#pragma unroll
    for (int w = 0; w < PARTS; ++w) {
      const float own = stats[(w * ROWS + r) * 2];
      const float f = own == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((own - most) * kLog2e);
      const float s = stats[(w * ROWS + r) * 2 + 1], v = parts[(w * ROWS + r) * PITCH + col];
      // a part that has seen only NaN has no maximum, and its sums count
      total += s == s ? s * f : s;
      value += v == v ? v * f : v;
    }
    const float result = total == 0.f ? 0.f : value / total;
    if (a.mask && (!attn_finite(result) || !attn_finite(total))) {
      atomicOr(&bad, 1u << r);
      continue;
    }
    const float2 sum = {most, total * __builtin_amdgcn_exp2f(-offset)};
    const int64_t flat = ((int64_t)at.batch * a.heads + h) * a.m + i;
    if (a.splits == 1) {
      (static_cast<T*>(a.O) + at.batch * a.o.batch + h * a.o.head + (int64_t)i * a.o.row)[col] = (T)result;
      if (col == 0 && a.lse) a.lse[flat] = attn_lse(sum);
    } else {
      a.part[(at.split * all + flat) * a.d + col] = result;
      if (col == 0) a.part_sum[at.split * all + flat] = sum;
    }
  }
  if (!a.mask) return;
  __syncthreads();
  for (unsigned left = uniform(bad); left; left &= left - 1) {
    const int r = __builtin_ctz(left), p = at.panel * ROWS + r, g = p / a.m, i = p - g * a.m, h = at.kv_head * a.group + g;
    if (r % kAttnWaves != uniform(tid >> 6)) continue;
    const int64_t flat = ((int64_t)at.batch * a.heads + h) * a.m + i;
    if (a.splits == 1) {
      const float2 sum = attn_exact_forward<T>(a, at.batch, h, i, begin, end,
                                               static_cast<T*>(a.O) + at.batch * a.o.batch + h * a.o.head + (int64_t)i * a.o.row, tid & 63);
      if ((tid & 63) == 0 && a.lse) a.lse[flat] = attn_lse(sum);
    } else {
      const float2 sum = attn_exact_forward<T>(a, at.batch, h, i, begin, end, a.part + (at.split * all + flat) * a.d, tid & 63);
      if ((tid & 63) == 0) a.part_sum[at.split * all + flat] = sum;
    }
  }
}

// The number N lanes on within 16.
template <int N> __device__ __forceinline__ float token_rotate(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
}

// More than 4 rows of a head of K and V, in half precision: 32 to a workgroup.  K and V are read once per 32 rows.  The four waves take
// blocks of 32 keys in turn, each with its own statistics, and no wave waits for another before the end.
template <int D, bool BIAS>
__global__ __launch_bounds__(256, D <= 64 ? 2 : 1) void attention_tokens_kernel(const AttnArgs a) {
  using T = _Float16;
  using Tile = AttnTile<D, 1>;
  constexpr int kBlock = 32 * Tile::kPitch;              // 32 keys or values of a wave
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  char* lds_k = lds_raw + wave * 2 * kBlock;
  char* lds_v = lds_k + kBlock;
  // the bias table of the group's heads, and the bucket of each relative position
  float* lds_table = reinterpret_cast<float*>(lds_raw + kAttnWaves * 2 * kBlock);
  int* lds_bucket = reinterpret_cast<int*>(lds_table + min(a.group, 32) * a.buckets);

  const TokenPanel<32> at(a);
  const int rows = at.rows, split = at.split, panel = at.panel, batch = at.batch, kv_head = at.kv_head;

  const int seen = a.lengths ? min(max(a.lengths[batch], 0), a.k) : a.k;
  const int blocks_all = (seen + 31) / 32;
  const int begin = (int)((int64_t)blocks_all * split / a.splits), end = (int)((int64_t)blocks_all * (split + 1) / a.splits);
  const int packed = panel * 32 + (lane & 31);
  const bool valid = packed < rows;
  const int of_group = valid ? packed / a.m : 0, row = valid ? packed - of_group * a.m : 0;
  const int head = kv_head * a.group + of_group;

  const T* Q = static_cast<const T*>(a.Q) + batch * a.q.batch + head * a.q.head + (int64_t)row * a.q.row;
  const T* K = static_cast<const T*>(a.K) + batch * a.kk.batch + kv_head * a.kk.head;
  const T* V = static_cast<const T*>(a.V) + batch * a.v.batch + kv_head * a.v.head;

  f32x16 acc[D / 32] = {};
  AttnRunning run;
  AttnStage<T, 32, Tile::kBytes, Tile::kPitch, 64> stage_k, stage_v;
  int t = begin + wave;
  if (t < end) {
    stage_k.load_block(K + (int64_t)t * 32 * a.kk.row, a.kk.row, seen - t * 32, a.d, lane);
    stage_v.load_block(V + (int64_t)t * 32 * a.v.row, a.v.row, seen - t * 32, a.d, lane);
  }
  AttnOwn<D, 1> q;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    q.v[0][s] = f16x8{};
    if (valid) q.v[0][s] = attn_load_piece<T>(Q, (2 * s + half) * 8, a.d);
  }
  if (a.scale < 0.f) q.negate();
  const float scale = fmaxf(fabsf(a.scale), kAttnLeastScale);
  const MaskLayout lay(a.m, a.k);
  int position = 0, first = 0;
  float low = 0.f, high = 0.f;                           // the bias at its ends
  const float* table = nullptr;
  if (BIAS) {
    const int head0 = panel * 32 / a.m;                  // of the group, the first one in this panel
    const int heads = min(a.group - head0, 32);
    const T* from = static_cast<const T*>(a.table) + (int64_t)(kv_head * a.group + head0) * a.buckets;
    for (int x = tid; x < heads * a.buckets; x += 256) lds_table[x] = (float)from[x];
    for (int x = tid; x < 2 * a.span + 1; x += 256) lds_bucket[x] = min(max(a.bucket_of[x], 0), a.buckets - 1);
    table = lds_table + (valid ? of_group - head0 : 0) * a.buckets;
    first = attn_position(a, batch);
    position = first + row;
    __syncthreads();
    low = table[lds_bucket[0]], high = table[lds_bucket[2 * a.span]];
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
      stage_k.load_block(K + (int64_t)t * 32 * a.kk.row, a.kk.row, seen - t * 32, a.d, lane);
      stage_v.load_block(V + (int64_t)t * 32 * a.v.row, a.v.row, seen - t * 32, a.d, lane);
    }
    unsigned word = ~0u;
    if (a.mask) word = valid ? (unsigned)(a.mask[lay.row_words + (int64_t)(key0 >> 6) * lay.ti * 64 + row] >> (key0 & 32)) : 0u;
    word &= attn_low_bits(seen - key0);
    if (!__any(word != 0)) continue;
    f32x16 x[1] = {};
    attn_product<Tile::kPitch>(x[0], lds_k, q, lane);
    if (BIAS && (key0 - (first + a.m - 1) >= a.span || key0 + 31 - first <= -a.span)) {
      attn_add_constant(x[0], scale, key0 > first ? high : low);      // each lane's own head
    } else if (BIAS) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int rel = key0 + 8 * (r / 4) + 4 * half + r % 4 - position;
        x[0][r] = __builtin_fmaf(x[0][r], scale, table[lds_bucket[min(max(rel, -a.span), a.span) + a.span]]);
      }
    }
    if (__any(word != ~0u)) attn_hide(x[0], word, half);
    attn_weights(x[0], run, attn_softmax_step<D, 1>(x, run, acc, AttnScores{scale, BIAS, 0.f}));
    attn_product_t<Tile::kPitch, D, 1>(acc, lds_v, x[0], lane);
  }

  // the four waves' parts, in LDS: [4][32][D + 1] sums, [4][32][2] statistics
  __syncthreads();
  float* lds_acc = reinterpret_cast<float*>(lds_raw);
  float* lds_stat = lds_acc + kAttnWaves * 32 * (D + 1);
  const float sum = attn_sum_halves(run.sum);
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
  token_finish<T, 32, kAttnWaves, D + 1>(a, at, lds_acc, lds_stat, kOffset, begin * 32, min(end * 32, seen), tid);
}

// x += 16 keys by 4 rows, 16 bytes of columns for each lane
__device__ __forceinline__ void token_scores(f32x4& x, const f32x4& k, const f32x4& q) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_4x4x1f32(k[e], q[e], x, 0, 0, 0);
}
__device__ __forceinline__ void token_scores(f32x4& x, const f16x8& k, const f16x8& q) {
  x = __builtin_amdgcn_mfma_f32_4x4x4f16(__builtin_shufflevector(k, k, 0, 1, 2, 3), __builtin_shufflevector(q, q, 0, 1, 2, 3), x, 0, 0, 0);
  x = __builtin_amdgcn_mfma_f32_4x4x4f16(__builtin_shufflevector(k, k, 4, 5, 6, 7), __builtin_shufflevector(q, q, 4, 5, 6, 7), x, 0, 0, 0);
}
// acc += columns by 4 rows, over the 16 keys
template <int GROUPS, int STEPS>
__device__ __forceinline__ void token_values(f32x4 (&acc)[GROUPS][STEPS][4], const f32x4 (&v)[4][STEPS], const f32x4 (&x)[GROUPS]) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < GROUPS; ++c) acc[c][s][e] = __builtin_amdgcn_mfma_f32_4x4x1f32(v[r][s][e], x[c][r], acc[c][s][e], 0, 0, 0);
}
template <int GROUPS, int STEPS>
__device__ __forceinline__ void token_values(f32x4 (&acc)[GROUPS][STEPS][8], const f16x8 (&v)[4][STEPS], const f32x4 (&x)[GROUPS]) {
  f16x4 p[GROUPS];
#pragma unroll
  for (int c = 0; c < GROUPS; ++c) p[c] = f16x4{(_Float16)x[c][0], (_Float16)x[c][1], (_Float16)x[c][2], (_Float16)x[c][3]};
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const f16x4 left = {v[0][s][e], v[1][s][e], v[2][s][e], v[3][s][e]};
#pragma unroll
      for (int c = 0; c < GROUPS; ++c) acc[c][s][e] = __builtin_amdgcn_mfma_f32_4x4x4f16(left, p[c], acc[c][s][e], 0, 0, 0);
    }
}
// The four sets of 16 lanes together, in all of them.
template <typename F> __device__ __forceinline__ float token_sets(float v, F both) {
  unsigned x = __builtin_bit_cast(unsigned, v);
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = __builtin_bit_cast(unsigned, both(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])));
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return both(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}

// Up to 4 rows of a head of K and V, and any number in single precision, on instructions that multiply 4 rows by 4 columns in each of
// sixteen blocks (4 x 1 by 1 x 4 fp32 numbers, or 4 x 4 by 4 x 4 fp16 ones): those of 32 x 32 do eight times the work for up to four rows.
//
// Lane l is row i = l % 4 of block l / 4 of the left operand and column i of that block of the right one.  Blocks split 16 keys into
// four sets g = l / 16 of four, and columns into quarters u = l / 4 % 4; E numbers are 16 bytes:
//   scores: lane l has 16 bytes of key 4 g + i, columns 4 E s + E u .., and of row i of Q the same columns.  Register r of the result,
//     added up over the quarters (lanes l, l + 4, l + 8, l + 12), is the score of key 4 g + r and row i;
//   values: those registers, as weights, are the right operand for keys 4 g + r; the left one are elements e of lane l's 16 bytes of V of
//     these keys, columns 16 E s + 4 E u + E i + e.  Register j of the result is column 16 E s + 4 E u + E j + e and row i, of set g.
// No number of K or V passes through LDS, and all loads are of 64 bytes and more at a time: bound by reading K and V (32 sequences of 3000
// states, 8 heads of 128 in fp32, 786 MB: 134 us, 5.9 TB/s; through LDS and instructions of 32 x 32 200 us).  Each set has statistics
// of its own.  ROWS: rows of the workgroup, four to each group of registers.
template <typename T, int D, int ROWS, bool BIAS>
__global__ __launch_bounds__(256, D <= 64 || ROWS <= 8 ? 2 : 1) void attention_token_kernel(const AttnArgs a) {
  using Piece = typename AttnPiece<T>::Type;
  constexpr int E = 16 / sizeof(T), kBlocks = sizeof(T) == 2 ? 2 : 1, kGroups = ROWS / 4, kScoreSteps = D / (4 * E), kValueSteps = (D + 16 * E - 1) / (16 * E);
  constexpr float kWeight = sizeof(T) == 2 ? kOffset : 0.f;
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), i = lane & 3, g = lane >> 4, u = lane >> 2 & 3;
  const TokenPanel<ROWS> at(a);
  const int batch = at.batch, kv_head = at.kv_head;
  const int seen = attn_seen(a, batch);
  // in units of 16 keys, kBlocks of which a wave takes at a time
  const int all = (seen + 16 * kBlocks - 1) / (16 * kBlocks), begin = (int)((int64_t)all * at.split / a.splits) * kBlocks,
            end = min((int)((int64_t)all * (at.split + 1) / a.splits) * kBlocks, (seen + 15) / 16);
  const T* K = static_cast<const T*>(a.K) + batch * a.kk.batch + kv_head * a.kk.head;
  const T* V = static_cast<const T*>(a.V) + batch * a.v.batch + kv_head * a.v.head;
  const bool whole = a.d % E == 0;

  Piece kf[kBlocks][kScoreSteps], vf[kBlocks][4][kValueSteps];
  // (rows behind the sequence's last are the last one again, with weights of 0)
  auto key_row = [&](int key) { return K + (int64_t)min(key, seen - 1) * a.kk.row; };
  auto value_row = [&](int key) { return V + (int64_t)min(key, seen - 1) * a.v.row; };
  // (one branch around all loads: with one around each, each would be waited for)
  auto load_keys = [&](int t) {
    if (whole) {
#pragma unroll
      for (int x = 0; x < kBlocks * kScoreSteps; ++x)
        kf[x / kScoreSteps][x % kScoreSteps] =
            attn_load_whole_piece<T>(key_row((t + x / kScoreSteps) * 16 + 4 * g + i), 4 * E * (x % kScoreSteps) + E * u, a.d);
    } else {
#pragma unroll
      for (int x = 0; x < kBlocks * kScoreSteps; ++x)
        kf[x / kScoreSteps][x % kScoreSteps] =
            attn_load_piece<T>(key_row((t + x / kScoreSteps) * 16 + 4 * g + i), 4 * E * (x % kScoreSteps) + E * u, a.d);
    }
  };
  auto load_values = [&](int t) {
    if (whole) {
#pragma unroll
      for (int x = 0; x < kBlocks * 4; ++x)
#pragma unroll
        for (int s = 0; s < kValueSteps; ++s)
          vf[x / 4][x % 4][s] = attn_load_whole_piece<T>(value_row((t + x / 4) * 16 + 4 * g + x % 4), 16 * E * s + 4 * E * u + E * i, a.d);
    } else {
#pragma unroll
      for (int x = 0; x < kBlocks * 4; ++x)
#pragma unroll
        for (int s = 0; s < kValueSteps; ++s)
          vf[x / 4][x % 4][s] = attn_load_piece<T>(value_row((t + x / 4) * 16 + 4 * g + x % 4), 16 * E * s + 4 * E * u + E * i, a.d);
    }
  };
  constexpr int kStep = kAttnWaves * kBlocks;
  int t = begin + wave * kBlocks;
  if (t < end) {
    load_keys(t);
    load_values(t);
  }

  Piece q[kGroups][kScoreSteps];
  int row[kGroups];
  const float* table[kGroups];
  float low[kGroups], high[kGroups];
  const float scale = a.scale;
  float* lds_table = reinterpret_cast<float*>(lds_raw);                   // the tables of the panel's heads, then the buckets
  int* lds_bucket = reinterpret_cast<int*>(lds_table + min(a.group, ROWS) * a.buckets);
  const int head0 = at.panel * ROWS / a.m;               // of the group, the first one in this panel
  int first = 0;
  if (BIAS) {
    const int heads = min(a.group - head0, ROWS);
    const T* from = static_cast<const T*>(a.table) + (int64_t)(kv_head * a.group + head0) * a.buckets;
    for (int x = tid; x < heads * a.buckets; x += 256) lds_table[x] = (float)from[x];
    for (int x = tid; x < 2 * a.span + 1; x += 256) lds_bucket[x] = min(max(a.bucket_of[x], 0), a.buckets - 1);
    first = attn_position(a, batch);
    __syncthreads();
  }
#pragma unroll
  for (int c = 0; c < kGroups; ++c) {
    const int packed = at.panel * ROWS + 4 * c + i;
    const bool valid = packed < at.rows;
    const int of_group = valid ? packed / a.m : head0;
    row[c] = valid ? packed - of_group * a.m : 0;
    const T* Q = static_cast<const T*>(a.Q) + batch * a.q.batch + (kv_head * a.group + of_group) * a.q.head + (int64_t)row[c] * a.q.row;
#pragma unroll
    for (int s = 0; s < kScoreSteps; ++s) q[c][s] = valid ? attn_load_piece<T>(Q, 4 * E * s + E * u, a.d) : Piece{};
    if (BIAS) {
      table[c] = lds_table + (of_group - head0) * a.buckets;
      low[c] = table[c][lds_bucket[0]], high[c] = table[c][lds_bucket[2 * a.span]];
    }
  }
  const MaskLayout lay(a.m, a.k);

  f32x4 acc[kGroups][kValueSteps][E] = {};
  float most[kGroups], sum[kGroups];
#pragma unroll
  for (int c = 0; c < kGroups; ++c) most[c] = -__builtin_inff(), sum[c] = 0.f;
  for (; t < end; t += kStep) {
    f32x4 x[kBlocks][kGroups] = {};
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int s = 0; s < kScoreSteps; ++s)
#pragma unroll
        for (int c = 0; c < kGroups; ++c) token_scores(x[n][c], kf[n][s], q[c][s]);
    if (t + kStep < end) load_keys(t + kStep);
#pragma unroll
    for (int c = 0; c < kGroups; ++c) {
      float top = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < kBlocks; ++n) {
        const int key0 = (t + n) * 16;
        unsigned word = attn_low_bits(seen - key0);
        if (a.mask && key0 < a.k) word &= (unsigned)(a.mask[lay.row_words + (int64_t)(key0 >> 6) * lay.ti * 64 + row[c]] >> (key0 & 63));
        word >>= 4 * g;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float s = x[n][c][r];
          s += token_rotate<4>(s);
          s += token_rotate<8>(s);
          s *= scale;
          if (BIAS) {
            const int rel = key0 + 4 * g + r - first - row[c];
            // far from the diagonal, where most keys are, the bias is one of two
            s += rel <= -a.span ? low[c] : rel >= a.span ? high[c] : table[c][lds_bucket[min(max(rel + a.span, 0), 2 * a.span)]];
          }
          s = (word >> r) & 1u ? s : -__builtin_inff();
          x[n][c][r] = s;
          top = fmaxf(top, s);
        }
      }
      if (__any(top > most[c])) {
        asm volatile("");
        const float now = fmaxf(most[c], top), factor = most[c] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((most[c] - now) * kLog2e);
        most[c] = now;
        sum[c] *= factor;
#pragma unroll
        for (int s = 0; s < kValueSteps; ++s)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[c][s][e] *= factor;
      }
      const float base = most[c] == -__builtin_inff() ? 0.f : most[c];
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[n][c][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][c][r] - base, kLog2e, kWeight));
          sum[c] += x[n][c][r];
        }
    }
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) token_values<kGroups, kValueSteps>(acc, vf[n], x[n]);
    if (t + kStep < end) load_values(t + kStep);
  }

  // the four sets of a wave, scaled to their common maximum; then the waves' parts in LDS: [4][ROWS][D] sums (rows 4 elements
  // apart from a multiple of the banks), [4][ROWS][2] statistics
  constexpr int kPitch = kValueSteps * 16 * E + 4;
  __syncthreads();
  float* lds_acc = reinterpret_cast<float*>(lds_raw);
  float* lds_stat = lds_acc + kAttnWaves * ROWS * kPitch;
#pragma unroll
  for (int c = 0; c < kGroups; ++c) {
    const float top = token_sets(most[c], [](float x, float y) { return fmaxf(x, y); });
    const float factor = most[c] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((most[c] - top) * kLog2e);
    const auto plus = [](float x, float y) { return x + y; };
    // (a set that has seen only NaN has no maximum, and its sums count)
    const float total = token_sets(sum[c] == sum[c] ? sum[c] * factor : sum[c], plus);
#pragma unroll
    for (int s = 0; s < kValueSteps; ++s)
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = acc[c][s][e][j];
          acc[c][s][e][j] = token_sets(v == v ? v * factor : v, plus);
        }
    // each set stores a register's part of the row
#pragma unroll
    for (int s = 0; s < kValueSteps; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (g == j) {
#pragma unroll
          for (int e = 0; e < E; e += 4) {
            const f32x4 v = {acc[c][s][e][j], acc[c][s][e + 1][j], acc[c][s][e + 2][j], acc[c][s][e + 3][j]};
            *reinterpret_cast<f32x4*>(lds_acc + (wave * ROWS + 4 * c + i) * kPitch + 16 * E * s + 4 * E * u + E * j + e) = v;
          }
        }
    if (lane < 4) {
      lds_stat[(wave * ROWS + 4 * c + i) * 2] = top;
      lds_stat[(wave * ROWS + 4 * c + i) * 2 + 1] = total;
    }
  }
  __syncthreads();
  token_finish<T, ROWS, kAttnWaves, kPitch>(a, at, lds_acc, lds_stat, kWeight, begin * 16, min(end * 16, seen), tid);
}

// Joins what the parts of the keys gave, by their sums.  16 lanes have four neighbouring elements each of a row; a row
// has LANES: where there are few rows, the 64 lanes of a wave, each 16 of which take every fourth part, else 16 (us, 64 and 16 lanes:
// 32768 rows of 64 columns, two parts 15.7 and 8.7; 8 rows of 128, 31 parts 10 and 13).  At most LANES parts.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnArgs a) {
  constexpr int kTurns = LANES / 16;
  const int64_t rows = (int64_t)a.batch * a.heads * a.m, flat = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (flat >= rows) return;
  const int lane = threadIdx.x % LANES, turn = lane >> 4;
  const float2 mine = lane < a.splits ? a.part_sum[lane * rows + flat] : float2{-__builtin_inff(), 0.f};
  float most = mine.x;
#pragma unroll
  for (int i = LANES / 2; i; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
  // (a part that has seen only NaN has no maximum, and its sum counts)
  const float share = mine.x == -__builtin_inff() ? mine.y : mine.y * __builtin_amdgcn_exp2f((mine.x - most) * kLog2e);
  float total = share;
#pragma unroll
  for (int i = LANES / 2; i; i >>= 1) total += __shfl_xor(total, i);
  const float weight = total == 0.f ? 0.f : share / total;
  const int i = (int)(flat % a.m);
  const int64_t bh = flat / a.m;
  const int h = (int)(bh % a.heads);
  T* O = static_cast<T*>(a.O) + bh / a.heads * a.o.batch + h * a.o.head + (int64_t)i * a.o.row;
  for (int c0 = 0; c0 < a.d; c0 += 64) {                  // every lane stays: the others read its weight
    const int c = c0 + lane % 16 * 4;
    f32x4 value = {};
    for (int s0 = 0; s0 < a.splits; s0 += 4 * kTurns) {   // four parts asked for at a time
      f32x4 v[4];
      attn_load_parts(v, a.part, a.splits, s0 + turn, kTurns, rows, flat, c, a.d);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = s0 + turn + u * kTurns;
        const float there = __shfl(weight, min(s, a.splits - 1), LANES), w = s < a.splits ? there : 0.f;
        if (w != 0.f) value += w * v[u];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (LANES == 64) {
        value[e] += __shfl_xor(value[e], 16);
        value[e] += __shfl_xor(value[e], 32);
      }
      if (turn == 0 && c + e < a.d) O[c + e] = (T)value[e];
    }
  }
  if (lane == 0 && a.lse) a.lse[flat] = attn_lse({most, total});
}

// Bits of the sparse matrix, from its CSR topology: the words by rows of ROWS rows at a time are made in LDS (which thread sets a bit first
// changes nothing) and written once, then one wave per tile of 64 x 64 turns its 64 words by rows into 64 by columns and marks the tile.
// Column indices out of range are passed over.  ROWS neighbouring words are one write, so as many rows as LDS has room for are taken;
// where one row has no room its entries are read once for each of its parts.  (Against bits set one by one in memory, us: 1.7 million entries of
// 4096 x 4096 26 / 95, 10.6 million of 12288 x 12288 99 / 520, 2 million of 2000 x 50000 56 / 121, 128000 of 64 x 200000 25 / 42.)
constexpr int kMaskWords = 8192;                          // of a workgroup
__global__ __launch_bounds__(256) void attention_mask_clear_kernel(int64_t words, uint64_t* mask) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) mask[i] = 0;
}
template <int ROWS>
__global__ __launch_bounds__(256) void attention_mask_rows_kernel(int m, int k, const int* __restrict__ row_offsets,
                                                                  const int* __restrict__ column_indices, uint64_t* mask) {
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  auto* bits = reinterpret_cast<unsigned long long*>(lds_raw);   // [word][row]
  constexpr int kEach = 256 / ROWS, kWords = kMaskWords / ROWS;
  const MaskLayout lay(m, k);
  const int parts = (int)((lay.tj + kWords - 1) / kWords), mine = threadIdx.x / kEach;
  for (int64_t id = blockIdx.x; id < lay.ti * (64 / ROWS) * parts; id += gridDim.x) {
    const int row0 = (int)(id / parts) * ROWS, row = row0 + mine, first = (int)(id % parts) * kWords, words = (int)min((int64_t)kWords, lay.tj - first);
    for (int i = threadIdx.x; i < words * ROWS; i += 256) bits[i] = 0;
    __syncthreads();
    if (row < m) {
      const int end = row_offsets[row + 1];
      for (int p = row_offsets[row] + threadIdx.x % kEach; p < end; p += kEach) {
        const int col = column_indices[p], word = (col >> 6) - first;
        if (col >= 0 && col < k && word >= 0 && word < words) atomicOr(bits + word * ROWS + mine, 1ull << (col & 63));
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < words * ROWS; i += 256)
      mask[lay.row_words + (int64_t)(first + i / ROWS) * lay.ti * 64 + row0 + i % ROWS] = bits[i];
    __syncthreads();
  }
}
__global__ __launch_bounds__(256) void attention_mask_tiles_kernel(int m, int k, uint64_t* mask) {
  const MaskLayout lay(m, k);
  const int lane = threadIdx.x & 63;
  for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < lay.ti * lay.tj; tile += (int64_t)gridDim.x * 4) {
    const int64_t ti = tile % lay.ti, tj = tile / lay.ti;
    const uint64_t word = mask[lay.row_words + (tj * lay.ti + ti) * 64 + lane];
    uint64_t column = 0;
    if (__any(word != 0)) {
#pragma unroll
      for (int b = 0; b < 64; ++b) {
        const uint64_t rows = __ballot((word >> b) & 1);
        if (lane == b) column = rows;
      }
      auto* marks = reinterpret_cast<unsigned long long*>(mask);
      if (lane == 0) {
        atomicOr(marks + lay.row_tiles + ti * ((lay.tj + 63) / 64) + (tj >> 6), 1ull << (tj & 63));
        atomicOr(marks + lay.col_tiles + tj * ((lay.ti + 63) / 64) + (ti >> 6), 1ull << (ti & 63));
      }
    }
    mask[lay.col_words + (ti * lay.tj + tj) * 64 + lane] = column;
  }
}

// The largest finite number of each sequence's head of K and V (of Q, dO: of all heads that share one), in up to 64 parts.
struct AttnOperand {
  const void* from;
  _Float16* to;
  AttnStrides s;
  int heads, group, rows;   // heads of K and V, and how many heads and rows of this operand belong to each
  int keys;                 // whether its rows are states, of which `lengths` counts
};
struct AttnOperands {
  AttnOperand of[4];
  int count, first, batch, kv_heads, d, k, parts;   // first: of Q, K, V, dO
  const int* lengths;
  float *most, *factors;    // [batch * kv_heads][4][parts], [batch * kv_heads][4]
};
__device__ __forceinline__ int64_t attn_operand_rows(const AttnOperands& o, const AttnOperand& x, int batch) {
  if (!x.keys) return (int64_t)x.group * x.rows;
  return o.lengths ? min(max(o.lengths[batch], 0), x.rows) : x.rows;
}
template <typename T>
__device__ __forceinline__ const T* attn_operand_row(const AttnOperand& x, int batch, int kv_head, int64_t r) {
  const int g = (int)(r / x.rows);
  return static_cast<const T*>(x.from) + batch * x.s.batch + ((int64_t)kv_head * x.group + g) * x.s.head + (r - (int64_t)g * x.rows) * x.s.row;
}
// Of rows [begin, end), by 256 threads, AHEAD pieces of 16 bytes each at a time (behind the last row that one again); no piece crosses a
// row's end, the last one of a row may overlap the one before.
template <int AHEAD>
__device__ __forceinline__ float attn_largest_of(const AttnOperands& o, const AttnOperand& x, int batch, int kv_head, int begin, int end) {
  const int pieces = (o.d + 3) / 4, row_step = 256 / pieces, piece_step = 256 % pieces;
  const float* base = static_cast<const float*>(x.from) + batch * x.s.batch + (int64_t)kv_head * x.group * x.s.head;
  int r = begin + threadIdx.x / pieces, c = threadIdx.x % pieces;
  auto next = [&]() {
    const int at = min(r, end - 1), g = x.group > 1 ? (unsigned)at / (unsigned)x.rows : 0;
    const float* row = base + g * x.s.head + (int64_t)(at - g * x.rows) * x.s.row + 4 * c;
    r += row_step;
    c += piece_step;
    if (c >= pieces) c -= pieces, ++r;
    return row;
  };
  float most = 0.f;
  while (r < end) {
    f32x4 v[AHEAD];
    if (o.d >= 4) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int back = max(4 * c + 4 - o.d, 0);
        v[i] = *reinterpret_cast<const AttnPiece<float>::Any*>(next() - back);
      }
    } else {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) v[i] = attn_load_piece<float>(next(), 0, o.d);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) most = attn_largest(most, v[i]);
  }
  return most;
}
__global__ __launch_bounds__(256) void attention_largest_kernel(const AttnOperands o) {
  __shared__ float waves[4];
  int64_t id = blockIdx.x;
  const int part = (int)(id % o.parts);
  id /= o.parts;
  const int which = (int)(id % o.count);
  id /= o.count;
  const int kv_head = (int)(id % o.kv_heads), batch = (int)(id / o.kv_heads);
  const AttnOperand& x = o.of[which];
  const int64_t rows = attn_operand_rows(o, x, batch);
  float most = attn_largest_of<4>(o, x, batch, kv_head, (int)(rows * part / o.parts), (int)(rows * (part + 1) / o.parts));
#pragma unroll
  for (int i = 32; i; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x == 0) o.most[(((int64_t)batch * o.kv_heads + kv_head) * 4 + which) * o.parts + part] = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
}
// Copies of the operands for the panel kernels, rows of D numbers, zeros behind d and behind a sequence's states.  Single precision:
// numbers times the power of two as two fp16 terms, the first ones of a row before the second ones.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_terms_kernel(const AttnOperands o, int64_t blocks, int each) {
  constexpr int kPieces = D / 8, kRows = 256 / kPieces;
  for (int id = blockIdx.y; id < each; id += gridDim.y) {
    const int which = id % o.count;
    const int64_t bh = id / o.count;
    const int kv_head = (int)(bh % o.kv_heads), batch = (int)(bh / o.kv_heads);
    const AttnOperand& x = o.of[which];
    const int64_t all = (int64_t)x.group * x.rows, rows = attn_operand_rows(o, x, batch);
    float factor = 1.f;
    if constexpr (sizeof(T) == 4) {
      const int lane = threadIdx.x & 63;
      float most = 0.f;
      if (o.most) {
        most = lane < o.parts ? o.most[(bh * 4 + which) * o.parts + lane] : 0.f;
      } else {                                            // few numbers: every workgroup looks at all of them
        most = attn_largest_of<8>(o, x, batch, kv_head, 0, (int)rows);
      }
#pragma unroll
      for (int i = 32; i; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
      if (!o.most) {
        __shared__ float waves[4];
        if (lane == 0) waves[threadIdx.x >> 6] = most;
        __syncthreads();
        most = fmaxf(fmaxf(waves[0], waves[1]), fmaxf(waves[2], waves[3]));
      }
      const int e = attn_exponent(most);
      factor = ldexpf(1.f, e);
      if (blockIdx.x == 0 && threadIdx.x == 0) o.factors[bh * 4 + o.first + which] = ldexpf(1.f, -e);
    }
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
      const int64_t r = block * kRows + threadIdx.x / kPieces;
      const bool mine = r < all && threadIdx.x < kRows * kPieces;
      const int c = threadIdx.x % kPieces * 8;
      _Float16* to = x.to + (bh * all + r) * (attn_terms<T>() * D) + c;
      if constexpr (sizeof(T) == 2) {
        f16x8 v = {};
        if (mine && r < rows) v = attn_load_piece<_Float16>(attn_operand_row<_Float16>(x, batch, kv_head, r), c, o.d);
        if (mine) *reinterpret_cast<f16x8*>(to) = v;
      } else {
        f16x8 hi = {}, lo = {};
        if (mine && r < rows) {
          const float* row = attn_operand_row<float>(x, batch, kv_head, r);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x4 v = attn_load_piece<float>(row, c + 4 * h, o.d) * factor;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              hi[4 * h + i] = (_Float16)v[i];
              lo[4 * h + i] = (_Float16)(v[i] - (float)hi[4 * h + i]);
            }
          }
        }
        if (mine) {
          *reinterpret_cast<f16x8*>(to) = hi;
          *reinterpret_cast<f16x8*>(to + D) = lo;
        }
      }
    }
    if (sizeof(T) == 4 && !o.most) __syncthreads();       // `waves` is read
  }
}

}  // namespace spdl
