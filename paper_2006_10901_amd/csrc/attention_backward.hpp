// Gradients of attention.  With P = exp(s - lse), D_i = dO_i . O_i and dS_ij = P_ij (dO_i . V_j - D_i):
//   dV_j = sum_i P_ij dO_i,   dK_j = scale sum_i dS_ij Q_i,   dQ_i = scale sum_j dS_ij K_j,   dtable[bucket] = sum of dS over its positions.
// Two kernels form the scores again, one by panels of queries (dQ, and D, which it leaves for the others), one by panels of keys (dK
// and dV): each sum has one owner, so that nothing is added up in an order that changes from call to call.  More workgroups of the
// second's launch go over the positions near the diagonal for the gradient of the bias, a sum per relative position.
#pragma once
#include "attention.hpp"

namespace spdl {

// The instructions take dS in fp16 terms, whose range it may leave either way (it is as large as dO and as small as a weight of a long
// row): it is taken times a power of two, the wave's own, lowered when a larger one comes along.  Numbers down to 2^-25 of the largest
// so far then keep all bits of a term.
struct AttnScale {
  float factor = 1.f, limit = 0.f;
  // makes room for x, which is taken times `by` already; what has been summed is scaled along.  Whether the factor has changed
  template <int BLOCKS> __device__ __forceinline__ bool fit(f32x16& x, f32x16 (&acc)[BLOCKS], float by) {
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(x[r]));
    if (!__any(most > limit * by)) return false;
    asm volatile("");
    // (a row of Inf makes no room for itself at the expense of the others)
    most = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, attn_finite(x[r]) ? fabsf(x[r]) : 0.f);
#pragma unroll
    for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if (!(most > limit * by)) return false;
    // 2^11 for the largest here, room for sixteen times as much; powers within +-100, so that the factors at the end are normal
    // numbers (a quotient that is not belongs to sums of less than 2^-126 of what comes)
    const int e = min(max(11 - ilogbf(fminf(most / by, 1e30f)), -100), 100);
    const float now = ldexpf(1.f, e), change = limit == 0.f ? 0.f : now / factor;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) acc[b] *= change;
    x *= now / by;
    factor = now;
    limit = 32768.f / now;
    return true;
  }
};

// Whether all relative positions of a block of 32 x 32 lie at the clamped ends of a bias; near: that of its first key and first query.
__device__ __forceinline__ bool attn_far(int near, int span) { return near - 31 >= span || near + 31 <= -span; }

// What a pass over a row's keys tells of the row: the sums of dS and of P over all of them and, for the gradient of the bias, over the
// blocks that lie at its lower and at its upper end (half precision: of P only there).  Added up in 64 bits: sums of thousands of terms that nearly cancel.
// `top`: what P is relative to, lse or (where lse is large, see attn_row_top) the largest score of those keys.
//
// P comes from lse, which is rounded to 2^-24 of itself: an error of up to 5e-7 (at an lse of 8) that all weights of a row share.  D is off by
// what rounding O cost.  But P adds up to 1 over a row, and dS to 0, so that the sums tell both errors: weights are P / sum P, and D
// is right once sum dS / sum P is added.  (Single precision: 9.2e-7 -> 4.7e-7 of dK's 2-norm.  Half precision with a bias: dtable's sums
// nearly cancel and were off by 3.8e-4 .. 1.2e-3, now 1.7e-4, what rounding the result costs.)
struct AttnRowSums { double ds, p, low, low_p, high, high_p; };
constexpr int kAttnRowSums = 7;                           // with the top
// Whether a call needs them for all rows.
template <typename T, bool BIAS> constexpr bool attn_row_sums() { return BIAS || sizeof(T) == 4; }

// (a row of Inf or NaN keeps its weights and its D)
__device__ __forceinline__ double attn_row_weight(double sum_p) { return sum_p > 0. && sum_p < 1e30 ? 1. / sum_p : 1.; }
// What the other kernels take of a row: D, what P is relative to, 1 / sum P and the sums of dS at the ends.
template <bool BIAS>
__device__ __forceinline__ void attn_finish_row(const AttnArgs& a, int64_t flat, float delta, const AttnRowSums& s, float top, double weight) {
  const double more = s.ds * weight;
  a.delta[flat] = more == more ? (float)(delta + more) : delta;
  a.top[flat] = top;
  a.weight[flat] = (float)weight;
  if constexpr (BIAS) {
    a.ends[2 * flat] = (float)(weight * (s.low - more * s.low_p));
    a.ends[2 * flat + 1] = (float)(weight * (s.high - more * s.high_p));
  }
}
template <bool BIAS> __device__ __forceinline__ AttnRowSums attn_row_sums_of(const AttnArgs& a, int64_t flat) {
  const int64_t rows = (int64_t)a.batch * a.heads * a.m;
  AttnRowSums s = {};
  for (int i0 = 0; i0 < a.splits; i0 += 4) {             // four parts asked for at a time, behind the last one that again
    double v[4][6];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int x = 0; x < (BIAS ? 6 : 2); ++x) v[u][x] = a.row_sums[(min(i0 + u, a.splits - 1) * rows + flat) * kAttnRowSums + x];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i0 + u >= a.splits) break;
      s.ds += v[u][0], s.p += v[u][1];
      if (BIAS) s.low += v[u][2], s.low_p += v[u][3], s.high += v[u][4], s.high_p += v[u][5];
    }
  }
  return s;
}

// Of 32 rows: whether weights of any of them take the long form (AttnScores); and whether their lse is why.
constexpr int kLarge = 1, kLargeLse = 2;

// A workgroup's panel of queries for the backward pass.
template <typename T, int D, bool BIAS> struct AttnQueries {
  static constexpr int kTerms = attn_terms<T>();
  AttnOwn<D, kTerms> q, g;
  float scale, lse, to_dp;
  bool large, large_lse;                                 // as kLarge, kLargeLse
  int64_t flat;
  // lse_of: lse, or each row's top
  __device__ __forceinline__ void load(const AttnArgs& a, const AttnPanelOf& at, const AttnFactors& f, const float* lse_of, int row, bool valid, int half) {
    flat = ((int64_t)at.batch * a.heads + at.head) * a.m + row;
    q.load(a.q16 + at.batch * a.q16s.batch + at.head * a.q16s.head, row * a.q16s.row, valid, a.width, half);
    g.load(a.g16 + at.batch * a.g16s.batch + at.head * a.g16s.head, row * a.g16s.row, valid, a.width, half);
    if (a.scale < 0.f) q.negate();
    scale = fmaxf(fabsf(a.scale) * (f.q * f.k), kAttnLeastScale);
    to_dp = f.g * f.v;
    lse = valid ? lse_of[flat] : -__builtin_inff();
    if (lse == -__builtin_inff()) lse = __builtin_inff();  // rows that see nothing, and those behind the last, have no weights
    large = large_lse = __any(attn_large(lse));
    if constexpr (BIAS) {
      // the bias's two ends
      const T* table = static_cast<const T*>(a.table) + (int64_t)at.head * a.buckets;
      const int first = a.bucket_of[0], last = a.bucket_of[2 * a.span];
      const float low = (float)table[min(max(first, 0), a.buckets - 1)], high = (float)table[min(max(last, 0), a.buckets - 1)];
      large |= !(fabsf(low) < kAttnLargeBias && fabsf(high) < kAttnLargeBias) || __any(attn_large(low - lse) || attn_large(high - lse));
    }
  }
  // Products become weights: without a bias, with one for all of them, or each with its own
  __device__ __forceinline__ void weights(f32x16& x) const {
    float shift = -lse * kLog2e;
    if (large) {
      // in place, as products that come to the same in the short form without a shift (a branch around both forms costs the registers of one of them)
      asm volatile("");
      const float inv = 1.f / scale;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = (__builtin_fmaf(x[r], scale, 0.f) - lse) * inv;
      shift = 0.f;
    }
    const float c = scale * kLog2e;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, shift));
  }
  __device__ __forceinline__ void weights(f32x16& x, float bias) const {
    if (!large) {
      const float c = scale * kLog2e, shift = (bias - lse) * kLog2e;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, shift));
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f((__builtin_fmaf(x[r], scale, bias) - lse) * kLog2e);
    }
  }
  __device__ __forceinline__ void weights(f32x16& x, const float* bias) const {
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f((__builtin_fmaf(x[r], scale, bias[8 * (r / 4) + r % 4]) - lse) * kLog2e);
  }
};

// Where lse is large, its rounding and that of the scores, which the forward pass may have added up in another order, are too: an lse of
// 1e9 is a multiple of 64.  The scores are then taken relative to the largest that the backward pass itself forms (a product has the same bits
// wherever it does) among the keys [begin, end), and weights over their sum.  A pass of its own over K, from memory, for the few calls that
// need it: in the kernel's own pass its registers would cost all others 12 % (fp16, 64 columns: 61 -> 69 us).
template <typename T, int D, bool BIAS>
__device__ __forceinline__ float2 attn_row_top(const AttnArgs& a, const AttnQueries<T, D, BIAS>& own, const AttnPanelOf& at, const _Float16* K, int row,
                                               bool valid, int begin, int end, int lane) {
  constexpr int kTerms = attn_terms<T>();
  const int half = lane >> 5;
  const MaskLayout lay(a.m, a.k);
  const int position = BIAS ? attn_position(a, at.batch) : 0;
  float top = -__builtin_inff(), sum = 0.f;
  for (int key0 = begin; key0 < end; key0 += 32) {
    const uint64_t word = attn_word(a.mask ? a.mask + lay.row_words + (int64_t)(key0 >> 6) * lay.ti * 64 : nullptr, row, valid);
    const unsigned w = ((unsigned)(word >> (key0 & 32)) & attn_low_bits(end - key0)) >> (4 * half);
    if (!__any(w != 0)) continue;
    AttnOwn<D, kTerms> k;
    k.load(K, min(key0 + (lane & 31), end - 1) * a.k16s.row, true, a.width, half);
    f32x16 x = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) attn_multiply<false>(x, k, own.q, s);
    float most = -__builtin_inff();
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float bias = 0.f;
      if (BIAS) {
        const int rel = key0 + 8 * (r / 4) + 4 * half + r % 4 - position - row;
        const int b = a.bucket_of[min(max(rel, -a.span), a.span) + a.span];
        bias = (float)static_cast<const T*>(a.table)[(int64_t)at.head * a.buckets + min(max(b, 0), a.buckets - 1)];
      }
      x[r] = attn_select(w, r, __builtin_fmaf(x[r], own.scale, bias), -__builtin_inff());
      most = fmaxf(most, x[r]);
    }
    const float now = fmaxf(top, attn_max_halves(most));
    if (now == -__builtin_inff()) continue;
    sum *= top == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((top - now) * kLog2e);
    top = now;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((x[r] - top) * kLog2e);
  }
  return {top, attn_sum_halves(sum)};
}

// Whether a row's weights are relative to the largest score instead of lse.
__device__ __forceinline__ bool attn_row_large(const AttnArgs& a, int batch, int head, int row) {
  const int blocks = (a.m + kAttnPanel - 1) / kAttnPanel * kAttnWaves;
  return a.large[((int64_t)batch * a.heads + head) * blocks + row / 32] & kLargeLse;
}

// dQ, by panels of 128 queries, and D = dO . O.
//
// Two workgroups to a compute unit, with 256 registers a thread, where that spills few of them (us, one -> two: fp16, 128 columns, 2 x 8 heads of
// 2048 x 2048 99 -> 74; fp32, 64 columns, 8 heads of 4096 x 4096 270 -> 207; but fp32 96 and 128 columns 93 -> 149 and 121 -> 237).
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256, (attn_queries_each<T, D>())) void attention_dq_kernel(const AttnArgs a) {
  constexpr int kTerms = attn_terms<T>();
  constexpr bool kSums = attn_row_sums<T, BIAS>();
  using Tile = AttnTile<D, kTerms, attn_queries_each<T, D>()>;
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  float* lds_bias = reinterpret_cast<float*>(lds_raw + Tile::kSets * Tile::kPair);

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
  AttnQueries<T, D, BIAS> own;
  own.load(a, at, f, a.lse, row, valid, half);
  float delta = 0.f;
  if (valid) {
    constexpr int kPiece = 16 / sizeof(T);
    const T* O = static_cast<const T*>(a.O) + batch * a.o.batch + head * a.o.head + (int64_t)row * a.o.row;
    const T* dO = static_cast<const T*>(a.dO) + batch * a.dout.batch + head * a.dout.head + (int64_t)row * a.dout.row;
    if (a.d % kPiece == 0) {
#pragma unroll 4
      for (int c = half * kPiece; c < a.d; c += 2 * kPiece) {
        const typename AttnPiece<T>::Type o = *reinterpret_cast<const typename AttnPiece<T>::Any*>(O + c),
                                          g = *reinterpret_cast<const typename AttnPiece<T>::Any*>(dO + c);
#pragma unroll
        for (int e = 0; e < kPiece; ++e) delta = __builtin_fmaf((float)o[e], (float)g[e], delta);
      }
    } else {
      for (int c = half; c < a.d; c += 2) delta = __builtin_fmaf((float)O[c], (float)dO[c], delta);
    }
  }
  delta = attn_sum_halves(delta);

  const MaskLayout lay(a.m, a.k);
  AttnSeenTiles tiles(a.mask, lay.row_tiles, lay.tj, lay.ti, first_row);
  int position = 0;
  if (BIAS) {
    attn_fill_bias<T, kAttnPadBlock>(lds_bias, a, head, tid, 256);
    position = attn_position(a, batch);
  }
  AttnRowSums sums = {};
  // Half precision: the rounding of O costs D as much as sqrt(keys) times what rounding dS costs, so that rows of few keys take D as
  // (sum P dP) / (sum P), from products formed twice, where all keys lie in one tile (2-norm of dQ, in units of what rounding it costs: 2 / 5 / 20
  // keys 2.5 / 1.7 / 1.48 with D = dO . O, 1.42 so; 65 1.46)
  const int only = kTerms == 1 ? tiles.only(wave >= 2, (seen + kAttnTile - 1) / kAttnTile) : -1;
  const bool tells = only < 0 ? at.split == 0 : begin <= only && only < end;   // the part of the keys that knows D
  // products become weights; whether the block lies at an end of the bias
  auto weigh = [&](f32x16& x, int near) {
    const bool far = BIAS && attn_far(near, a.span);
    if constexpr (!BIAS) own.weights(x);
    else if (far) own.weights(x, lds_bias[near > 0 ? 2 * a.span + kAttnPadBlock : kAttnPadBlock]);
    else own.weights(x, lds_bias + kAttnPadBlock + a.span + near - (lane & 31) + 4 * half);
    return far;
  };
  const int64_t rows = (int64_t)a.batch * a.heads * a.m;
  double* row_sums = a.row_sums + (at.split * rows + own.flat) * kAttnRowSums;      // where there are splits
  if (at.split == 0 && lane == 0) a.large[(((int64_t)batch * a.heads + head) * at.panels + at.panel) * kAttnWaves + wave] = own.large_lse ? kLargeLse : own.large ? kLarge : 0;
  if (own.large_lse) {
    asm volatile("");
    const float2 top = attn_row_top<T, D, BIAS>(a, own, at, K, row, valid, begin * kAttnTile, min(end * kAttnTile, seen), lane);
    // (rows of Inf or NaN keep what they have, those that see none of these keys need none; lanes of a row store the same)
    if (attn_finite(own.lse) && attn_finite(top.x)) own.lse = top.x;
    if (valid && kTerms == 1) {
      if (a.splits == 1) a.weight[own.flat] = (float)attn_row_weight(top.y);
      else row_sums[1] = top.y;
    }
    if (valid && a.splits > 1) row_sums[6] = top.x;
  }
  float to_ds = own.to_dp, delta_ds = delta, from_ds = 1.f;   // what makes dS, taken times the factor of ds_scale

  f32x16 acc[D / 32] = {};
  AttnScale ds_scale;
  typename Tile::template Stage<kAttnTile, 256> stage_k, stage_v;
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
    char* lds_k = lds_raw + set * Tile::kPair;
    char* lds_v = lds_k + kAttnTile * Tile::kPitch;
    if (Tile::kSets == 1) __syncthreads();
    stage_k.store(lds_k, tid);
    stage_v.store(lds_v, tid);
    const int key0 = t * kAttnTile;
    const uint64_t word = attn_first(word_next, seen - key0);
    __syncthreads();
    t = tiles.next(t + 1, end);
    if (t < end) load(t);
    if (wave_row >= a.m || !__any(word != 0)) continue;
    const bool hide = __any(word != ~0ull);
    if (kTerms == 1 && key0 == only * kAttnTile) {
      float sum_p = 0.f, sum = 0.f;
#pragma unroll 1
      for (int b = 0; b < 2; ++b) {
        f32x16 x = {}, y = {};
        attn_product<Tile::kPitch>(x, lds_k + b * 32 * Tile::kPitch, own.q, lane);
        attn_product<Tile::kPitch>(y, lds_v + b * 32 * Tile::kPitch, own.g, lane);
        weigh(x, key0 + 32 * b - (position + wave_row));
        const unsigned w = (unsigned)(word >> (32 * b)) >> (4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sum_p += attn_select(w, r, x[r], 0.f);
          sum += attn_select(w, r, x[r] * y[r], 0.f);
        }
      }
      sum_p = attn_sum_halves(sum_p);
      sum = attn_sum_halves(sum) * own.to_dp;
      if (sum_p > 0.f) delta = sum / sum_p;
      delta_ds = delta * ds_scale.factor;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int near = key0 + 32 * b - (position + wave_row);   // relative position of the block's first key and first query
      f32x16 x = {}, y = {};
      attn_product<Tile::kPitch>(x, lds_k + b * 32 * Tile::kPitch, own.q, lane);
      attn_product<Tile::kPitch>(y, lds_v + b * 32 * Tile::kPitch, own.g, lane);
      __builtin_amdgcn_s_setprio(1);                       // as in the forward pass (fp32 202 -> 194 us)
      const bool far = weigh(x, near);
      const unsigned w = (unsigned)(word >> (32 * b)) >> (4 * half);
      const bool sum_weights = kTerms == 2 || far;
      if (hide && sum_weights) {
        asm volatile("");
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = attn_select(w, r, x[r], 0.f);
      }
      float sum = 0.f, sum_p = 0.f;
      if (sum_weights) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sum_p += x[r];
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] *= __builtin_fmaf(y[r], to_ds, -delta_ds);
      if (hide) {                                          // whatever stands where the row does not look
        asm volatile("");
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = attn_select(w, r, x[r], 0.f);
      }
      if (kSums) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += x[r];
      }
      if (kSums) {
        sum *= from_ds;
        sums.ds += sum;
        sums.p += sum_p;
        if (BIAS && far) {
          (near > 0 ? sums.high : sums.low) += sum;
          (near > 0 ? sums.high_p : sums.low_p) += sum_p;
        }
      }
      if (ds_scale.fit(x, acc, ds_scale.factor)) to_ds = own.to_dp * ds_scale.factor, delta_ds = delta * ds_scale.factor, from_ds = 1.f / ds_scale.factor;
      attn_product_t<Tile::kPitch, D, kTerms>(acc, lds_k + b * 32 * Tile::kPitch, x, lane);
      __builtin_amdgcn_s_setprio(0);
    }
  }

  // a row that sees nothing: its dS of 0 times Inf or NaN of states that its neighbours see is NaN, and so may D be
  const bool none = own.lse == __builtin_inff();
  if (none) {
    delta = 0.f;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) acc[b] = f32x16{};
  }
  double weight = 1.;                                    // what the row's P is taken times
  double s[6] = {sums.ds, sums.p, sums.low, sums.low_p, sums.high, sums.high_p};
  if constexpr (kSums) {
#pragma unroll
    for (int i = 0; i < 6; ++i) s[i] += __shfl_xor(s[i], 32);
  }
  const AttnRowSums all = {s[0], s[1], s[2], s[3], s[4], s[5]};
  if (a.splits == 1) {
    if (kTerms == 2) weight = attn_row_weight(all.p);
    else if (own.large_lse && valid) weight = a.weight[own.flat];
    if (valid && half == 0) attn_finish_row<BIAS>(a, own.flat, delta, all, none ? -__builtin_inff() : own.lse, weight);
  } else if (valid && half == 0) {
    if (tells) a.delta[own.flat] = delta;
#pragma unroll
    for (int i = 0; i < 6; ++i)
      if ((BIAS || i < 2) && !(kTerms == 1 && i == 1 && own.large_lse)) row_sums[i] = s[i];
  }
  if (a.mask) {
    // (rows whose own numbers are Inf or NaN are right as they are, and so are those that see nothing)
    const unsigned bad = attn_not_finite(acc, false) & (unsigned)__ballot(valid && attn_finite(own.lse) && attn_finite(delta));
    if (lane == 0) a.again[blockIdx.x * kAttnWaves + wave] = bad;
  }
  const float factor = (float)weight * a.scale * f.k / ds_scale.factor;
  if (a.splits == 1) {
    T* dQ = static_cast<T*>(a.dQ) + batch * a.dq.batch + head * a.dq.head + (int64_t)row * a.dq.row;
    attn_store_rows<T, D>(dQ, valid, acc, factor, a.d, half);
  } else {
    attn_store_rows<float, D>(a.part + (at.split * rows + own.flat) * a.d, valid, acc, factor, a.d, half);
  }
}
// Runs before the parts are added up: they are sums of P as lse gives it, with D as it is then.
template <typename T>
__global__ __launch_bounds__(256) void attention_dq_again_kernel(const AttnArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  unsigned left = uniform(a.again[blockIdx.x * kAttnWaves + wave]);
  if (!left) return;
  const AttnPanelOf at(a, a.m);
  int begin, end;
  const int seen = attn_seen(a, at.batch);
  attn_tiles_of_split(a, at.split, seen, begin, end);
  for (; left; left &= left - 1) {
    const int row = at.panel * kAttnPanel + wave * 32 + __builtin_ctz(left);
    const int64_t flat = ((int64_t)at.batch * a.heads + at.head) * a.m + row;
    const float delta = a.delta[flat], weight = a.splits == 1 ? a.weight[flat] : 1.f;
    const float lse = a.splits == 1 ? a.top[flat] : attn_row_large(a, at.batch, at.head, row)
                          ? (float)a.row_sums[((int64_t)at.split * a.batch * a.heads * a.m + flat) * kAttnRowSums + 6] : a.lse[flat];
    if (a.splits == 1)
      attn_exact_dq<T>(a, at.batch, at.head, row, begin * kAttnTile, min(end * kAttnTile, seen), lse, delta, weight,
                       static_cast<T*>(a.dQ) + at.batch * a.dq.batch + at.head * a.dq.head + (int64_t)row * a.dq.row, lane);
    else
      attn_exact_dq<T>(a, at.batch, at.head, row, begin * kAttnTile, min(end * kAttnTile, seen), lse, delta, weight,
                       a.part + ((int64_t)at.split * a.batch * a.heads * a.m + flat) * a.d, lane);
  }
}

// Sums of dS by relative position, a wave's own: x holds keys in its registers and queries in its lanes.  The block of 32 x 32 goes through
// LDS by diagonals: key j and query i at row j - i + 31 and column i of 63 rows, whose other places stay 0, and lane l adds up row l.  Each
// relative position between the clamped ends then has one lane that adds it.
constexpr int kAttnDiagonalPitch = 36, kAttnDiagonalBlock = 63 * kAttnDiagonalPitch;      // floats per wave
__device__ __forceinline__ void attn_sum_diagonals(const f32x16& x, float* block, float* sums, int near, int span, double& low, double& high, int lane) {
  float* at = block + (4 * (lane >> 5) - (lane & 31) + 31) * kAttnDiagonalPitch + (lane & 31);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int r = 0; r < 16; ++r) at[(8 * (r / 4) + r % 4) * kAttnDiagonalPitch] = x[r];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const float* row = block + min(lane, 62) * kAttnDiagonalPitch;
  f32x4 s = {};
#pragma unroll
  for (int i = 0; i < 32; i += 4) s += *reinterpret_cast<const f32x4*>(row + i);
  const float sum = (s[0] + s[1]) + (s[2] + s[3]);
  const int rel = near + lane - 31;                       // of row `lane`
  if (lane < 63) {
    if (rel <= -span) low += sum;
    else if (rel >= span) high += sum;
    else sums[rel + span] += sum;
  }
}

// The gradient of the bias by relative position, by panels of 128 queries: the blocks near the diagonal are formed again, with the
// right D; what lies at the ends of the bias attention_dq_kernel has summed by rows.
template <typename T, int D>
__device__ __forceinline__ void attn_dbias(const AttnArgs& a, char* lds_raw) {
  constexpr int kTerms = attn_terms<T>();
  using Tile = AttnTile<D, kTerms, attn_keys_each<T, D>()>;
  float* lds_bias = reinterpret_cast<float*>(lds_raw + Tile::kPair);
  float* lds_blocks = lds_bias + (attn_bias_entries(a.span, kAttnPadBlock) + 3) / 4 * 4;
  float* lds_sums = lds_blocks + kAttnWaves * kAttnDiagonalBlock;
  const int n = 2 * a.span + 1;

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  const AttnPanelOf at(a, a.m, a.bias_splits, blockIdx.x - a.bias_from, gridDim.x - a.bias_from);
  const int batch = at.batch, head = at.head, kv_head = at.kv_head;
  const int seen = attn_seen(a, batch);
  const int first_row = at.panel * kAttnPanel, wave_row = first_row + wave * 32, row = wave_row + (lane & 31);
  const bool valid = row < a.m;
  const int position = attn_position(a, batch);
  // tiles that hold relative positions between the ends
  const int lowest = position + first_row - a.span - kAttnTile, highest = position + first_row + kAttnPanel + a.span;
  const int from = max(lowest, 0) / kAttnTile, to = max(from, min((seen + kAttnTile - 1) / kAttnTile, max(highest, 0) / kAttnTile + 1));
  const int begin = from + (to - from) * at.split / a.bias_splits, end = from + (to - from) * (at.split + 1) / a.bias_splits;

  const _Float16* K = a.k16 + batch * a.k16s.batch + kv_head * a.k16s.head;
  const _Float16* V = a.v16 + batch * a.v16s.batch + kv_head * a.v16s.head;
  const AttnFactors f = attn_factors<T>(a, batch, kv_head);
  AttnQueries<T, D, true> own;
  own.load(a, at, f, a.top, row, valid, half);
  attn_fill_bias<T, kAttnPadBlock>(lds_bias, a, head, tid, 256);
  float* sums = lds_sums + wave * n;
  float* block = lds_blocks + wave * kAttnDiagonalBlock;
  for (int x = lane; x < n; x += 64) sums[x] = 0.f;
  for (int x = lane; x < kAttnDiagonalBlock; x += 64) block[x] = 0.f;

  float delta = 0.f, weight = 1.f;
  double low = 0., high = 0.;
  if (valid) {
    delta = a.delta[own.flat];
    weight = a.weight[own.flat];
    if (half == 0 && at.split == 0) low = a.ends[2 * own.flat], high = a.ends[2 * own.flat + 1];
  }

  const MaskLayout lay(a.m, a.k);
  AttnSeenTiles tiles(a.mask, lay.row_tiles, lay.tj, lay.ti, first_row);
  typename Tile::template Stage<kAttnTile, 256> stage_k, stage_v;
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
  while (t < end) {
    char* lds_k = lds_raw;
    char* lds_v = lds_k + kAttnTile * Tile::kPitch;
    __syncthreads();
    stage_k.store(lds_k, tid);
    stage_v.store(lds_v, tid);
    const int key0 = t * kAttnTile;
    const uint64_t word = valid ? attn_first(word_next, seen - key0) : 0ull;     // (a diagonal's sum takes in lanes behind the last row)
    __syncthreads();
    t = tiles.next(t + 1, end);
    if (t < end) load(t);
    if (wave_row >= a.m || !__any(word != 0)) continue;
    for (int b = 0; b < 2; ++b) {
      const int near = key0 + 32 * b - (position + wave_row);
      if (attn_far(near, a.span)) continue;
      f32x16 x = {}, y = {};
      attn_product<Tile::kPitch>(x, lds_k + b * 32 * Tile::kPitch, own.q, lane);
      attn_product<Tile::kPitch>(y, lds_v + b * 32 * Tile::kPitch, own.g, lane);
      own.weights(x, lds_bias + kAttnPadBlock + a.span + near - (lane & 31) + 4 * half);
      const unsigned w = (unsigned)(word >> (32 * b)) >> (4 * half);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = attn_select(w, r, x[r] * weight * __builtin_fmaf(y[r], own.to_dp, -delta), 0.f);
      attn_sum_diagonals(x, block, sums, near, a.span, low, high, lane);
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    low += __shfl_xor(low, o);
    high += __shfl_xor(high, o);
  }
  if (lane == 0) {
    sums[0] += (float)low;
    sums[2 * a.span] += (float)high;
  }
  __syncthreads();
  float* sum_to = a.part_bias + ((((int64_t)head * a.batch + batch) * at.panels + at.panel) * a.bias_splits + at.split) * n;
  for (int x = tid; x < n; x += 256) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) s += lds_sums[w * n + x];
    sum_to[x] = s;
  }
}

// dK and dV, by panels of 128 keys: a wave has 32 of them, tiles of 64 queries, of every head that shares the keys, are shared by the waves.
// LARGE: all weights in the long form (AttnScores), and taken over their rows' sums in half precision as well.
template <typename T, int D, bool BIAS, bool LARGE>
__device__ __forceinline__ void attn_dkv(const AttnArgs& a, char* lds_raw, int split, int panel, int batch, int kv_head) {
  constexpr int kTerms = attn_terms<T>();
  constexpr bool kWeights = kTerms == 2 || LARGE;
  using Tile = AttnTile<D, kTerms, attn_keys_each<T, D>()>;
  float* lds_stats = reinterpret_cast<float*>(lds_raw + Tile::kSets * Tile::kPair);     // of each set, 64 times: lse (as an exponent of 2; with
  // a bias lse itself), D, what P is taken times, and the exponents with the bias's two ends
  float* lds_bias = lds_stats + Tile::kSets * 5 * kAttnTile;

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  const int seen = attn_seen(a, batch);
  const int first_key = panel * kAttnPanel, wave_key = first_key + wave * 32, key = wave_key + (lane & 31);
  const bool valid = key < seen;
  const int tiles = (a.m + kAttnTile - 1) / kAttnTile;
  // the tiles of all heads of the group, one after the other, are dealt to the splits in runs: from tile t of head h on, up to that of `last`
  const int64_t all = first_key < seen ? (int64_t)a.group * tiles : 0, begin = all * split / a.splits, end = all * (split + 1) / a.splits;
  int h = tiles ? (int)(begin / tiles) : 0, t = (int)(begin - (int64_t)h * tiles);
  const int last_h = tiles ? (int)(end / tiles) : 0, last_t = (int)(end - (int64_t)last_h * tiles);

  const _Float16* Q = a.q16 + batch * a.q16s.batch + (int64_t)kv_head * a.group * a.q16s.head;
  const _Float16* dO = a.g16 + batch * a.g16s.batch + (int64_t)kv_head * a.group * a.g16s.head;
  const int64_t stat0 = ((int64_t)batch * a.heads + (int64_t)kv_head * a.group) * a.m;

  AttnOwn<D, kTerms> kf, vf;
  kf.load(a.k16 + batch * a.k16s.batch + kv_head * a.k16s.head, key * a.k16s.row, valid, a.width, half);
  vf.load(a.v16 + batch * a.v16s.batch + kv_head * a.v16s.head, key * a.v16s.row, valid, a.width, half);
  if (a.scale < 0.f) kf.negate();
  const AttnFactors f = attn_factors<T>(a, batch, kv_head);
  const float scale = fmaxf(fabsf(a.scale) * (f.q * f.k), kAttnLeastScale), to_dp = f.g * f.v, c = scale * kLog2e;

  const MaskLayout lay(a.m, a.k);
  AttnSeenTiles seen_tiles(a.mask, lay.col_tiles, lay.ti, lay.tj, first_key);
  const int position = BIAS ? attn_position(a, batch) : 0;

  // from there on the next that the panel takes part in; whether there is one
  auto next = [&]() {
    while (h < last_h || (h == last_h && t < last_t)) {
      const int stop = h == last_h ? last_t : tiles;
      t = seen_tiles.next(t, stop);
      if (t < stop) return true;
      ++h;
      t = 0;
    }
    return false;
  };

  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  AttnScale ds_scale;
  typename Tile::template Stage<kAttnTile, 256> stage_q, stage_g;
  // (one address for a wave: chosen lane by lane in the loop it was itself loaded, and waited for, in every tile: 98 -> 94 us)
  const float* stats_of = (wave == 0 ? LARGE ? a.top : a.lse : wave == 1 ? a.delta : a.weight) + stat0;
  float stat = 0.f;
  const auto whole_q = stage_q.whole_offsets(a.q16s.row, tid);
  const auto whole_g = stage_g.whole_offsets(a.g16s.row, tid);
  uint64_t word_next = 0;
  auto load = [&]() {
    const int rows = a.m - t * kAttnTile;
    word_next = attn_word(a.mask ? a.mask + lay.col_words + (int64_t)t * lay.tj * 64 : nullptr, key, valid);
    stage_q.load(Q + h * a.q16s.head + (int64_t)t * kAttnTile * a.q16s.row, a.q16s.row, rows, a.width, whole_q, tid);
    stage_g.load(dO + h * a.g16s.head + (int64_t)t * kAttnTile * a.g16s.row, a.g16s.row, rows, a.width, whole_g, tid);
    if (wave < (kWeights ? 3 : 2)) stat = lane < rows ? stats_of[(int64_t)h * a.m + t * kAttnTile + lane] : wave == 0 ? -__builtin_inff() : 0.f;
  };
  bool more = next();
  int bias_head = -1;
  float low = 0.f, high = 0.f;                            // the bias at its ends
  if (more) load();
  for (int set = 0; more; set ^= Tile::kSets - 1) {
    char* lds_q = lds_raw + set * Tile::kPair;
    char* lds_g = lds_q + kAttnTile * Tile::kPitch;
    float* lds_lse = lds_stats + set * 5 * kAttnTile;
    float* lds_delta = lds_lse + kAttnTile;
    float* lds_weight = lds_delta + kAttnTile;
    float* lds_ends = lds_weight + kAttnTile;
    if (Tile::kSets == 1) __syncthreads();
    stage_q.store(lds_q, tid);
    stage_g.store(lds_g, tid);
    const int row0 = t * kAttnTile;
    const uint64_t word = valid ? word_next : 0ull;
    if (BIAS && h != bias_head) {
      __syncthreads();                                    // the head before may still be at work
      attn_fill_bias<T, kAttnPadBlock>(lds_bias, a, kv_head * a.group + h, tid, 256);
      __syncthreads();
      bias_head = h;
      low = lds_bias[kAttnPadBlock], high = lds_bias[2 * a.span + kAttnPadBlock];
    }
    if (tid < 64) {
      // rows that see nothing, and those behind the last, have no weights
      const float l = stat == -__builtin_inff() ? __builtin_inff() : stat;
      lds_lse[tid] = BIAS || LARGE ? l : kOffset - l * kLog2e;
      if (BIAS) {
        lds_ends[tid] = __builtin_fmaf(low - l, kLog2e, kOffset);
        lds_ends[64 + tid] = __builtin_fmaf(high - l, kLog2e, kOffset);
      }
    } else if (tid < (kWeights ? 192 : 128)) {
      lds_lse[tid] = stat;
    }
    __syncthreads();
    ++t;
    more = next();
    if (more) load();
    if (!__any(word != 0)) continue;
    const bool hide = __any(word != ~0ull);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int near = wave_key - (position + row0 + 32 * b);
      f32x16 x = {}, y = {};
      attn_product<Tile::kPitch, true>(x, lds_q + b * 32 * Tile::kPitch, kf, lane);
      attn_product<Tile::kPitch>(y, lds_g + b * 32 * Tile::kPitch, vf, lane);
      __builtin_amdgcn_s_setprio(1);                       // as in the forward pass (fp32 202 -> 194 us)
      if (!LARGE && (!BIAS || attn_far(near, a.span))) {
        const float* shifts = (BIAS ? lds_ends + (near > 0 ? 64 : 0) : lds_lse) + b * 32 + half * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, shifts[8 * (r / 4) + r % 4]));
      } else {
        // the table's entries are read one by one, so that far positions of a large bias read its end
        const int rel = near + (lane & 31) - 4 * half + a.span;
        const float* l = lds_lse + b * 32 + half * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float bias = BIAS ? lds_bias[kAttnPadBlock + min(max(rel - (8 * (r / 4) + r % 4), 0), 2 * a.span)] : 0.f;
          x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(__builtin_fmaf(x[r], scale, bias) - l[8 * (r / 4) + r % 4], kLog2e, kOffset));
        }
      }
      if constexpr (kWeights) {
        const float* weights = lds_weight + b * 32 + half * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] *= weights[8 * (r / 4) + r % 4];
      }
      if (hide) {
        asm volatile("");
        const unsigned w = (unsigned)(word >> (32 * b)) >> (4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          x[r] = attn_select(w, r, x[r], 0.f);
          y[r] = attn_select(w, r, y[r], 0.f);
        }
      }
      const float* deltas = lds_delta + b * 32 + half * 4;
#pragma unroll
      for (int r = 0; r < 16; ++r) y[r] = x[r] * __builtin_fmaf(y[r], to_dp, -deltas[8 * (r / 4) + r % 4]);
      attn_product_t<Tile::kPitch, D, kTerms>(dv, lds_g + b * 32 * Tile::kPitch, x, lane);
      if (!ds_scale.fit(y, dk, 1.f)) y *= ds_scale.factor;
      attn_product_t<Tile::kPitch, D, kTerms>(dk, lds_q + b * 32 * Tile::kPitch, y, lane);
      __builtin_amdgcn_s_setprio(0);
    }
  }

  // states behind the sequence's last: the weights of 0 that their lanes have times Inf or NaN of Q, dO or D are NaN
  if (!valid) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b) dk[b] = dv[b] = f32x16{};
  }
  const float offset = __builtin_amdgcn_exp2f(-kOffset);
  const float to_dk = a.scale * f.q * offset / ds_scale.factor, to_dv = f.g * offset;
  const bool stored = key < a.k;
  if (a.mask) {
    const unsigned bad = (attn_not_finite(dk, false) | attn_not_finite(dv, false)) & (unsigned)__ballot(valid);
    if (lane == 0) a.again[blockIdx.x * kAttnWaves + wave] = bad;
  }
  if (a.splits == 1) {
    T* dK = static_cast<T*>(a.dK) + batch * a.dk.batch + kv_head * a.dk.head + (int64_t)key * a.dk.row;
    T* dV = static_cast<T*>(a.dV) + batch * a.dv.batch + kv_head * a.dv.head + (int64_t)key * a.dv.row;
    attn_store_rows<T, D>(dK, stored, dk, to_dk, a.d, half);
    attn_store_rows<T, D>(dV, stored, dv, to_dv, a.d, half);
  } else {
    const int64_t rows = (int64_t)a.batch * a.kv_heads * a.k, flat = ((int64_t)batch * a.kv_heads + kv_head) * a.k + key;
    attn_store_rows<float, D>(a.part + (split * rows + flat) * a.d, stored, dk, to_dk, a.d, half);
    attn_store_rows<float, D>(a.part + ((a.splits + split) * rows + flat) * a.d, stored, dv, to_dv, a.d, half);
  }
}
// Two workgroups to a compute unit as for dQ (fp32, 64 columns 369 -> 292 us, fp16 96 106 -> 98), but not at 128 columns (fp16 143 -> 235).
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256, (attn_keys_each<T, D>())) void attention_dkv_kernel(const AttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  if (BIAS && (int)blockIdx.x >= a.bias_from) {
    attn_dbias<T, D>(a, lds_raw);
    return;
  }
  const int panels = (a.k + kAttnPanel - 1) / kAttnPanel;
  const AttnPlace place(a, panels * a.splits, blockIdx.x, BIAS ? a.bias_from : gridDim.x);
  // One answer for all rows of the heads, and two copies of the kernel: with a branch in each block the short form takes longer
  // (fp16, us: 64 columns, 8 x 16 heads of 512 x 2048 94 -> 98, 96 and 128 columns, 2 x 8 heads of 2048 x 2048 68 -> 73 and 122 -> 126).
  const int blocks = a.group * ((a.m + kAttnPanel - 1) / kAttnPanel) * kAttnWaves, *of = a.large + ((int64_t)place.batch * a.kv_heads + place.kv_head) * blocks;
  int any = 0;
  for (int i = threadIdx.x & 63; i < blocks; i += 64) any |= of[i];
  const int split = place.piece % a.splits, panel = place.piece / a.splits;
  if (__builtin_expect(__any(any), 0)) attn_dkv<T, D, BIAS, true>(a, lds_raw, split, panel, place.batch, place.kv_head);
  else attn_dkv<T, D, BIAS, false>(a, lds_raw, split, panel, place.batch, place.kv_head);
}
template <typename T>
__global__ __launch_bounds__(256) void attention_dkv_again_kernel(const AttnArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  unsigned left = uniform(a.again[blockIdx.x * kAttnWaves + wave]);
  if (!left) return;
  const int panels = (a.k + kAttnPanel - 1) / kAttnPanel;
  const AttnPlace place(a, panels * a.splits);
  const int split = place.piece % a.splits, panel = place.piece / a.splits;
  const int64_t all = (int64_t)a.group * ((a.m + kAttnTile - 1) / kAttnTile), begin = all * split / a.splits, end = all * (split + 1) / a.splits;
  for (; left; left &= left - 1) {
    const int key = panel * kAttnPanel + wave * 32 + __builtin_ctz(left);
    if (a.splits == 1) {
      T* dK = static_cast<T*>(a.dK) + place.batch * a.dk.batch + place.kv_head * a.dk.head + (int64_t)key * a.dk.row;
      T* dV = static_cast<T*>(a.dV) + place.batch * a.dv.batch + place.kv_head * a.dv.head + (int64_t)key * a.dv.row;
      attn_exact_dkv<T>(a, place.batch, place.kv_head, key, begin, end, dK, dV, lane);
    } else {
      const int64_t rows = (int64_t)a.batch * a.kv_heads * a.k, flat = ((int64_t)place.batch * a.kv_heads + place.kv_head) * a.k + key;
      float *dK = a.part + (split * rows + flat) * a.d, *dV = a.part + ((a.splits + split) * rows + flat) * a.d;
      attn_exact_dkv<T>(a, place.batch, place.kv_head, key, begin, end, dK, dV, lane);
    }
  }
}

// Adds up what `splits` workgroups left of each of the rows, in their order: of one array, or of two that lie one behind the other; a
// thread has four neighbouring elements of a row.
struct AttnSum { AttnStrides to; void* out; };
template <typename T>
__device__ __forceinline__ void attn_add_parts(int splits, int64_t rows, int heads, int per_head, int d, const float* part, int64_t flat, int c, float weight,
                                               const AttnSum& x) {
  f32x4 s = {};
  for (int i0 = 0; i0 < splits; i0 += 4) {
    f32x4 v[4];
    attn_load_parts(v, part, splits, i0, 1, rows, flat, c, d);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u < splits) s += v[u];
  }
  s *= weight;
  const int64_t bh = flat / per_head;
  T* row = static_cast<T*>(x.out) + bh / heads * x.to.batch + bh % heads * x.to.head + (flat % per_head) * x.to.row;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c + e < d) row[c + e] = (T)s[e];
}
// Of dQ, whose rows' sums over their keys are added up and put to use here (SUMS).
template <typename T, bool BIAS, bool SUMS>
__global__ __launch_bounds__(256) void attention_sum_dq_kernel(const AttnArgs a) {
  const int pieces = (a.d + 3) / 4;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)a.batch * a.heads * a.m;
  if (at >= rows * pieces) return;
  const int64_t flat = at / pieces;
  const bool first = at % pieces == 0;
  const int c = (int)(at % pieces) * 4, i = (int)(flat % a.m);
  const int64_t bh = flat / a.m;
  if (attn_row_large(a, (int)(bh / a.heads), (int)(bh % a.heads), i)) {
    // parts relative to the largest score of each
    auto sum_of = [&](int s, int x) { return a.row_sums[(s * rows + flat) * kAttnRowSums + x]; };
    // (that of NaN stays as it is: its parts have no scale)
    const float lse = a.lse[flat];
    float top = -__builtin_inff();
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, (float)sum_of(s, 6));
    const bool scaled = attn_finite(lse) && attn_finite(top);
    AttnRowSums all = {};
    f32x4 value = {};
    for (int s = 0; s < a.splits; ++s) {
      const float own = (float)sum_of(s, 6);
      const double factor = !scaled ? 1. : own == -__builtin_inff() ? 0. : (double)__builtin_amdgcn_exp2f((own - top) * kLog2e);
      if (factor == 0.) continue;
      value += (float)factor * attn_load_piece<float>(a.part + (s * rows + flat) * a.d, c, a.d);
      all.p += factor * sum_of(s, 1);
      if (SUMS) all.ds += factor * sum_of(s, 0);
      if (BIAS) all.low += factor * sum_of(s, 2), all.low_p += factor * sum_of(s, 3), all.high += factor * sum_of(s, 4), all.high_p += factor * sum_of(s, 5);
    }
    const double w = attn_row_weight(all.p);
    if (first) attn_finish_row<BIAS>(a, flat, a.delta[flat], all, scaled ? top : lse, w);
    T* row = static_cast<T*>(a.dQ) + bh / a.heads * a.dq.batch + bh % a.heads * a.dq.head + (int64_t)i * a.dq.row;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < a.d) row[c + e] = (T)(value[e] * (float)w);
    return;
  }
  float weight = 1.f;
  if (SUMS && (sizeof(T) == 4 || first)) {
    const AttnRowSums s = attn_row_sums_of<BIAS>(a, flat);
    const double w = sizeof(T) == 4 ? attn_row_weight(s.p) : 1.;
    weight = (float)w;
    if (first) attn_finish_row<BIAS>(a, flat, a.delta[flat], s, a.lse[flat], w);
  } else if (first) {
    a.top[flat] = a.lse[flat];
    a.weight[flat] = 1.f;
  }
  attn_add_parts<T>(a.splits, rows, a.heads, a.m, a.d, a.part, flat, c, weight, AttnSum{a.dq, a.dQ});
}

// dtable of one head: the panels' sums by relative position (runs of panels by as many groups of threads as 1024 allow, added up in their
// order), then those of a bucket, in ascending position, 8 to 64 threads to a bucket.
template <typename T>
__device__ __forceinline__ void attn_dtable(const AttnArgs& a, int head, int parts, T* dtable, char* lds_raw) {
  const int n = 2 * a.span + 1, groups = n < 1024 ? 1024 / n : 1;
  double* sums = reinterpret_cast<double*>(lds_raw);      // [groups][n], then [n] in the first
  int* buckets = reinterpret_cast<int*>(sums + groups * n);
  const float* from = a.part_bias + (int64_t)head * parts * n;
  for (int at = threadIdx.x; at < groups * n; at += 1024) {
    const int group = at / n, x = at - group * n, end = (int)((int64_t)parts * (group + 1) / groups);
    const int bucket = a.bucket_of[x];
    double s = 0.;
    for (int i0 = (int)((int64_t)parts * group / groups); i0 < end; i0 += 16) {   // sixteen asked for at a time
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = from[(int64_t)min(i0 + u, end - 1) * n + x];
#pragma unroll
      for (int u = 0; u < 16; ++u)
        if (i0 + u < end) s += v[u];
    }
    sums[at] = s;
    if (group == 0) buckets[x] = min(max(bucket, 0), a.buckets - 1);
  }
  __syncthreads();
  for (int x = threadIdx.x; x < n; x += 1024) {
    double s = sums[x];
    for (int g = 1; g < groups; ++g) s += sums[g * n + x];
    sums[x] = s;
  }
  __syncthreads();
  const int each = a.buckets <= 16 ? 64 : a.buckets <= 32 ? 32 : a.buckets <= 64 ? 16 : 8, b = threadIdx.x / each, part = threadIdx.x % each;
  double s = 0.;
#pragma unroll 4
  for (int x = n * part / each; x < n * (part + 1) / each; ++x) s += buckets[x] == b ? sums[x] : 0.;
  for (int o = 1; o < each; o <<= 1) s += __shfl_xor(s, o);
  if (part == 0 && b < a.buckets) dtable[(int64_t)head * a.buckets + b] = (T)s;
}

// What is left when the panels are done: dtable, a workgroup per head (`tables` of them), and dK and dV added up where they were split.
template <typename T>
__global__ __launch_bounds__(1024) void attention_finish_kernel(const AttnArgs a, int tables, int parts, T* dtable) {
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  if ((int)blockIdx.x < tables) {
    attn_dtable<T>(a, blockIdx.x, parts, dtable, lds_raw);
    return;
  }
  const int pieces = (a.d + 3) / 4;
  const int64_t rows = (int64_t)a.batch * a.kv_heads * a.k, all = rows * pieces;
  int64_t at = (int64_t)(blockIdx.x - tables) * 1024 + threadIdx.x;
  if (at >= 2 * all) return;
  const bool behind = at >= all;
  if (behind) at -= all;
  attn_add_parts<T>(a.splits, rows, a.kv_heads, a.k, a.d, a.part + (behind ? a.splits * rows * a.d : 0), at / pieces, (int)(at % pieces) * 4, 1.f,
                    behind ? AttnSum{a.dv, a.dV} : AttnSum{a.dk, a.dK});
}

}  // namespace spdl
