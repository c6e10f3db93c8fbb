// Gradients of attention.  With P = exp(s - lse), D_i = dO_i . O_i and dS_ij = P_ij (dO_i . V_j - D_i):
//   dV_j = sum_i P_ij dO_i,   dK_j = scale sum_i dS_ij Q_i,   dQ_i = scale sum_j dS_ij K_j,   dtable[bucket] = sum of dS over its positions.
// Two kernels form the scores again, one by panels of queries (dQ, the bias, and D, which it leaves for the other), one by panels of
// keys (dK and dV): each sum has one owner, so that nothing is added up in an order that changes from call to call.
#pragma once
#include "attention.hpp"

namespace spdl {

// fp16 instructions take dS in half precision, whose range it may leave either way (it is as large as dO and as small as a weight
// of a long row): it is taken times a power of two, the wave's own, lowered when a larger one comes along.  Numbers down to 2^-25 of
// the largest so far then keep all their bits.
struct AttnScale {
  float factor = 1.f, limit = 0.f;
  // makes room for x; what has been summed is scaled along
  template <int BLOCKS> __device__ __forceinline__ void fit(const f32x16& x, f32x16 (&acc)[BLOCKS]) {
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(x[r]));
    if (__any(most > limit)) {
#pragma unroll
      for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
      // 2^11 for the largest here, room for sixteen times as much; powers within +-100, so that the factors at the end are normal
      // numbers (a quotient that is not belongs to sums of less than 2^-126 of what comes)
      const int e = min(max(11 - ilogbf(fminf(most, 1e30f)), -100), 100);
      const float now = ldexpf(1.f, e), change = limit == 0.f ? 0.f : now / factor;
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) acc[b] *= change;
      factor = now;
      limit = 32768.f / now;
    }
  }
};

template <typename T, int BLOCKS> __device__ __forceinline__ void attn_fit(AttnScale& s, f32x16& x, f32x16 (&acc)[BLOCKS]) {
  if constexpr (sizeof(T) == 2) {
    s.fit(x, acc);
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] *= s.factor;
  }
}

// Sums of dS by relative position, a wave's own: x holds keys in its registers and queries in its lanes.  The block of 32 x 32 goes
// through LDS, and lane l sums the l-th diagonal.  Each relative position between the clamped ends then has one lane that adds it.
__device__ __forceinline__ void attn_sum_diagonals(const f32x16& x, float* block, float* sums, int near, int span, float& low, float& high,
                                                   int lane) {
  const int half = lane >> 5;
  if (near - 31 >= span || near + 31 <= -span) {          // all of it beyond an end
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s += x[r];
    if (near > 0) high += s;
    else low += s;
    return;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int r = 0; r < 16; ++r) block[(lane & 31) * 33 + 8 * (r / 4) + 4 * half + r % 4] = x[r];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int off = lane - 31;                              // key minus query within the block
  float s = 0.f;
  for (int i = 0; i < 32; ++i) {
    const int j = i + off;
    if (j >= 0 && j < 32) s += block[i * 33 + j];
  }
  const int rel = near + off;
  if (lane < 63) {
    if (rel <= -span) low += s;
    else if (rel >= span) high += s;
    else sums[rel + span] += s;
  }
}

constexpr int kAttnDiagBytes = 32 * 33 * 4;               // per wave

// dQ, by panels of 128 queries, and D = dO . O.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256) void attention_dq_kernel(const AttnArgs a) {
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
  const int64_t flat = ((int64_t)batch * a.heads + head) * a.m + row;

  const T* Q = static_cast<const T*>(a.Q) + batch * a.q.batch + head * a.q.head;
  const T* K = static_cast<const T*>(a.K) + batch * a.kk.batch + kv_head * a.kk.head;
  const T* V = static_cast<const T*>(a.V) + batch * a.v.batch + kv_head * a.v.head;
  const T* O = static_cast<const T*>(a.O) + batch * a.o.batch + head * a.o.head;
  const T* dO = static_cast<const T*>(a.dO) + batch * a.dout.batch + head * a.dout.head;

  AttnOwn<T, D> q, g;
  float delta = 0.f;
  {
    AttnOwn<T, D> o;
    attn_load_own<T, D>(o, O + (int64_t)row * a.o.row, valid, a.d, half);
    attn_load_own<T, D>(g, dO + (int64_t)row * a.dout.row, valid, a.d, half);
#pragma unroll
    for (int s = 0; s < Tile::kSteps; ++s)
#pragma unroll
      for (int e = 0; e < Tile::kPiece; ++e) delta = __builtin_fmaf((float)o[s][e], (float)g[s][e], delta);
    delta += attn_other_half(delta);
  }
  if (valid && half == 0 && split == 0) a.delta[flat] = delta;
  attn_load_own<T, D>(q, Q + (int64_t)row * a.q.row, valid, a.d, half);
  if (a.scale < 0.f) {
#pragma unroll
    for (int s = 0; s < Tile::kSteps; ++s) q[s] = -q[s];
  }
  const float scale = fabsf(a.scale);
  const float c = BIAS ? kLog2e : scale * kLog2e;
  float lse = valid ? a.lse[flat] : 0.f;
  if (lse == -__builtin_inff()) lse = __builtin_inff();   // a row that sees nothing has no weights
  const float shift = BIAS ? lse : -lse * kLog2e;

  const MaskLayout lay(a.m, a.k);
  const uint64_t *tiles_a = nullptr, *tiles_b = nullptr;
  if (a.mask) {
    const int64_t per = (lay.tj + 63) / 64;
    tiles_a = a.mask + lay.row_tiles + (int64_t)(first_row >> 6) * per;
    if ((first_row >> 6) + 1 < lay.ti) tiles_b = tiles_a + per;
  }
  int position = 0;
  float *diag_block = nullptr, *diag_sums = nullptr, low = 0.f, high = 0.f;
  if (BIAS) {
    attn_fill_bias<T>(lds_bias, a, head, tid, 256);
    position = attn_position(a, batch);
    if (a.part_bias) {
      float* after = lds_bias + attn_bias_entries(a.span);
      diag_block = after + wave * (32 * 33);
      diag_sums = after + kAttnWaves * (32 * 33) + wave * (2 * a.span + 1);
      for (int x = lane; x < 2 * a.span + 1; x += 64) diag_sums[x] = 0.f;
    }
  }

  f32x16 acc[D / 32] = {};
  AttnScale ds_scale;
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
    if (wave_row >= a.m || !__any(word != 0)) continue;
    const bool hide = __any(word != ~0ull);
    const int near = key0 - (position + wave_row);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 x = {}, y = {};
      attn_product<D>(x, lds_k + b * 32 * Tile::kPitch, q, lane);
      attn_product<D>(y, lds_v + b * 32 * Tile::kPitch, g, lane);
      if (BIAS) {
        if (near - 31 >= a.span || near + 63 <= -a.span) {
          const float far = lds_bias[near > 0 ? 2 * a.span + kAttnPad : kAttnPad];
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, far);
        } else {
          const float* at = lds_bias + kAttnPad + a.span + near + 32 * b - (lane & 31) + 4 * half;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, at[8 * (r / 4) + r % 4]);
        }
      }
      const unsigned w = (unsigned)(word >> (32 * b)) >> (4 * half);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = BIAS ? __builtin_amdgcn_exp2f((x[r] - shift) * c) : __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, shift));
        x[r] = p * (y[r] - delta);
        if (hide) x[r] = attn_bit(w, r) ? x[r] : 0.f;
      }
      if (BIAS && a.part_bias) attn_sum_diagonals(x, diag_block, diag_sums, near + 32 * b, a.span, low, high, lane);
      attn_fit<T>(ds_scale, x, acc);
      attn_product_t<D>(acc, lds_k + b * 32 * Tile::kPitch, x, lane, T{});
    }
  }

  const float factor = a.scale / ds_scale.factor;
  if (a.splits == 1) {
    T* dQ = static_cast<T*>(a.dQ) + batch * a.dq.batch + head * a.dq.head + (int64_t)row * a.dq.row;
    attn_store_rows<T, D>(dQ, valid, acc, factor, a.d, half);
  } else {
    const int64_t rows = (int64_t)a.batch * a.heads * a.m;
    attn_store_rows<float, D>(a.part + (split * rows + flat) * a.d, valid, acc, factor, a.d, half);
  }
  if (BIAS && a.part_bias) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
      low += __shfl_xor(low, o);
      high += __shfl_xor(high, o);
    }
    if (lane == 0) {
      diag_sums[0] += low;
      diag_sums[2 * a.span] += high;
    }
    __syncthreads();
    const int n = 2 * a.span + 1;
    const float* from = lds_bias + attn_bias_entries(a.span) + kAttnWaves * (32 * 33);
    float* to = a.part_bias + (((int64_t)head * a.batch + batch) * panels * a.splits + panel * a.splits + split) * n;
    for (int x = tid; x < n; x += 256) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kAttnWaves; ++w) s += from[w * n + x];
      to[x] = s;
    }
  }
}

// dK and dV, by panels of 128 keys: a wave has 32 of them, tiles of 64 queries, of every head that shares the keys, are shared by the waves.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(256) void attention_dkv_kernel(const AttnArgs a) {
  using Tile = AttnTile<T, D>;
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  char* lds_q = lds_raw;
  char* lds_g = lds_raw + kAttnTile * Tile::kPitch;
  float* lds_lse = reinterpret_cast<float*>(lds_raw + 2 * kAttnTile * Tile::kPitch);
  float* lds_delta = lds_lse + kAttnTile;
  float* lds_bias = lds_delta + kAttnTile;

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = uniform(tid >> 6);
  const int panels = (a.k + kAttnPanel - 1) / kAttnPanel;
  int work = attn_work(blockIdx.x, gridDim.x);
  const int split = work % a.splits;
  work /= a.splits;
  const int panel = work % panels;
  work /= panels;
  const int batch = work % a.batch, kv_head = work / a.batch;

  const int seen = a.lengths ? min(max(a.lengths[batch], 0), a.k) : a.k;
  const int first_key = panel * kAttnPanel, wave_key = first_key + wave * 32, key = wave_key + (lane & 31);
  const bool valid = key < seen;
  const int tiles = (a.m + kAttnTile - 1) / kAttnTile;
  // the tiles of all heads of the group, one after the other, are dealt to the splits in runs
  const int64_t all = (int64_t)a.group * tiles;
  const int64_t begin = first_key < seen ? all * split / a.splits : 0, end = first_key < seen ? all * (split + 1) / a.splits : 0;

  const T* K = static_cast<const T*>(a.K) + batch * a.kk.batch + kv_head * a.kk.head;
  const T* V = static_cast<const T*>(a.V) + batch * a.v.batch + kv_head * a.v.head;
  const T* Q = static_cast<const T*>(a.Q) + batch * a.q.batch + (int64_t)kv_head * a.group * a.q.head;
  const T* dO = static_cast<const T*>(a.dO) + batch * a.dout.batch + (int64_t)kv_head * a.group * a.dout.head;
  const int64_t stat0 = ((int64_t)batch * a.heads + (int64_t)kv_head * a.group) * a.m;

  AttnOwn<T, D> kf, vf;
  attn_load_own<T, D>(kf, K + (int64_t)key * a.kk.row, valid, a.d, half);
  attn_load_own<T, D>(vf, V + (int64_t)key * a.v.row, valid, a.d, half);
  if (a.scale < 0.f) {
#pragma unroll
    for (int s = 0; s < Tile::kSteps; ++s) kf[s] = -kf[s];
  }
  const float scale = fabsf(a.scale);
  const float c = BIAS ? kLog2e : scale * kLog2e;

  const MaskLayout lay(a.m, a.k);
  const uint64_t *tiles_a = nullptr, *tiles_b = nullptr;
  if (a.mask) {
    const int64_t per = (lay.ti + 63) / 64;
    tiles_a = a.mask + lay.col_tiles + (int64_t)(first_key >> 6) * per;
    if ((first_key >> 6) + 1 < lay.tj) tiles_b = tiles_a + per;
  }
  const int position = BIAS ? attn_position(a, batch) : 0;

  // the next (head of the group, tile of queries) that the panel takes part in
  auto next = [&](int64_t at) {
    while (at < end) {
      const int h = (int)(at / tiles), t = (int)(at - (int64_t)h * tiles);
      const int stop = (int)min((int64_t)tiles, end - (int64_t)h * tiles);
      const int n = attn_next_tile(t, stop, tiles_a, tiles_b);
      if (n < stop) return (int64_t)h * tiles + n;
      at = (int64_t)h * tiles + stop;
    }
    return end;
  };

  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  AttnScale ds_scale;
  AttnStage<T, D, kAttnTile, 256> stage_q, stage_g;
  float stat = 0.f;
  auto load = [&](int64_t at) {
    const int h = (int)(at / tiles), t = (int)(at - (int64_t)h * tiles), rows = a.m - t * kAttnTile;
    stage_q.load(Q + h * a.q.head + (int64_t)t * kAttnTile * a.q.row, a.q.row, rows, a.d, tid);
    stage_g.load(dO + h * a.dout.head + (int64_t)t * kAttnTile * a.dout.row, a.dout.row, rows, a.d, tid);
    const int r = tid & 63;
    if (tid < 128) stat = r < rows ? (tid < 64 ? a.lse : a.delta)[stat0 + (int64_t)h * a.m + t * kAttnTile + r] : tid < 64 ? -__builtin_inff() : 0.f;
  };
  int64_t at = next(begin);
  int bias_head = -1;
  if (at < end) load(at);
  while (at < end) {
    __syncthreads();
    stage_q.store(lds_q, tid);
    stage_g.store(lds_g, tid);
    const int h = (int)(at / tiles), row0 = (int)(at - (int64_t)h * tiles) * kAttnTile;
    if (tid < 64) {
      // rows that see nothing, and those behind the last, have no weights
      const float l = stat == -__builtin_inff() ? __builtin_inff() : stat;
      lds_lse[tid] = BIAS ? l : AttnType<T>::kOffset - l * kLog2e;
    } else if (tid < 128) {
      lds_delta[tid - 64] = stat;
    }
    if (BIAS && h != bias_head) {
      attn_fill_bias<T>(lds_bias, a, kv_head * a.group + h, tid, 256);
      bias_head = h;
    }
    __syncthreads();
    at = next(at + 1);
    if (at < end) load(at);
    uint64_t word = valid ? ~0ull : 0ull;
    if (a.mask && valid) word = a.mask[lay.col_words + (int64_t)(row0 >> 6) * lay.tj * 64 + key];
    if (!__any(word != 0)) continue;
    const bool hide = __any(word != ~0ull);
    const int near = wave_key - (position + row0);        // relative position of the wave's first key and the tile's first query
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 x = {}, y = {};
      attn_product<D>(x, lds_q + b * 32 * Tile::kPitch, kf, lane);
      attn_product<D>(y, lds_g + b * 32 * Tile::kPitch, vf, lane);
      if (BIAS) {
        if (near - 63 >= a.span || near + 31 <= -a.span) {
          const float far = lds_bias[near > 0 ? 2 * a.span + kAttnPad : kAttnPad];
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, far);
        } else {
          const float* from = lds_bias + kAttnPad + a.span + near - 32 * b + (lane & 31) - 4 * half;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __builtin_fmaf(x[r], scale, from[-(8 * (r / 4) + r % 4)]);
        }
      }
      const unsigned w = (unsigned)(word >> (32 * b)) >> (4 * half);
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(lds_lse + b * 32 + q4 * 8 + half * 4);
        const f32x4 dl = *reinterpret_cast<const f32x4*>(lds_delta + b * 32 + q4 * 8 + half * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * q4 + e;
          float p = BIAS ? __builtin_amdgcn_exp2f(__builtin_fmaf(x[r] - l[e], c, AttnType<T>::kOffset))
                         : __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, l[e]));
          float s = p * (y[r] - dl[e]);
          if (hide) {
            p = attn_bit(w, r) ? p : 0.f;
            s = attn_bit(w, r) ? s : 0.f;
          }
          x[r] = p;
          y[r] = s;
        }
      }
      attn_product_t<D>(dv, lds_g + b * 32 * Tile::kPitch, x, lane, T{});
      attn_fit<T>(ds_scale, y, dk);
      attn_product_t<D>(dk, lds_q + b * 32 * Tile::kPitch, y, lane, T{});
    }
  }

  const float offset = __builtin_amdgcn_exp2f(-AttnType<T>::kOffset);
  const bool stored = key < a.k;
  if (a.splits == 1) {
    T* dK = static_cast<T*>(a.dK) + batch * a.dk.batch + kv_head * a.dk.head + (int64_t)key * a.dk.row;
    T* dV = static_cast<T*>(a.dV) + batch * a.dv.batch + kv_head * a.dv.head + (int64_t)key * a.dv.row;
    attn_store_rows<T, D>(dK, stored, dk, a.scale / ds_scale.factor * offset, a.d, half);
    attn_store_rows<T, D>(dV, stored, dv, offset, a.d, half);
  } else {
    const int64_t rows = (int64_t)a.batch * a.kv_heads * a.k, flat = ((int64_t)batch * a.kv_heads + kv_head) * a.k + key;
    attn_store_rows<float, D>(a.part + (split * rows + flat) * a.d, stored, dk, a.scale / ds_scale.factor * offset, a.d, half);
    attn_store_rows<float, D>(a.part + ((a.splits + split) * rows + flat) * a.d, stored, dv, offset, a.d, half);
  }
}

// Adds up what `splits` workgroups left of each of the rows, in their order.
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_kernel(int splits, int64_t rows, int heads, int per_head, int d, const float* part,
                                                            AttnStrides to, T* out) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= rows * d) return;
  const int64_t flat = at / d;
  const int col = (int)(at - flat * d);
  float s = 0.f;
  for (int i = 0; i < splits; ++i) s += part[(int64_t)i * rows * d + at];
  const int64_t bh = flat / per_head;
  out[bh / heads * to.batch + bh % heads * to.head + (flat % per_head) * to.row + col] = (T)s;
}

// dtable of one head: the workgroups' sums by relative position, in their order, then those of a bucket, in ascending position.
template <typename T>
__global__ __launch_bounds__(1024) void attention_dtable_kernel(const AttnArgs a, int parts, T* dtable) {
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  float* sums = reinterpret_cast<float*>(lds_raw);
  const int n = 2 * a.span + 1, head = blockIdx.x;
  const float* from = a.part_bias + (int64_t)head * parts * n;
  for (int x = threadIdx.x; x < n; x += 1024) {
    float s = 0.f;
    for (int i = 0; i < parts; ++i) s += from[(int64_t)i * n + x];
    sums[x] = s;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < a.buckets; b += 1024) {
    float s = 0.f;
    for (int x = 0; x < n; ++x)
      if (min(max(a.bucket_of[x], 0), a.buckets - 1) == b) s += sums[x];
    dtable[(int64_t)head * a.buckets + b] = (T)s;
  }
}

}  // namespace spdl
