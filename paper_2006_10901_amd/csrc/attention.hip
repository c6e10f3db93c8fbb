// Attention over the positions of a sparse matrix, or all: argument checks, the choice of kernel and of how the work is split, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/spdl.h"
#include "attention_backward.hpp"
#include "attention_forward.hpp"

namespace {

using namespace spdl;

constexpr int kMostRows = 1 << 29;
constexpr int kMostWidth = 128;

struct Plan {
  bool token;                          // the kernel for a few queries, and how many rows its workgroups take
  int token_rows;
  int forward_splits, dq_splits, dkv_splits, dbias_splits;
  int64_t forward_blocks, dq_blocks, dkv_blocks;      // without the splits
  int64_t rows, kv_rows, parts;        // parts: workgroups that leave sums of dS per head
  int width;                           // d rounded up to the width of a kernel
  bool copied;                         // whether the panel kernels take copies of Q, K, V and dO: fp16 terms of fp32 numbers, or rows
                                       // of whole 16-byte pieces where the caller's are not, or lie 2^24 elements apart
  int most_parts;
  // offsets into the workspace, in bytes; the terms of Q, K, V and dO and their factors come first (single precision)
  int64_t most, factors, q16, k16, v16, g16;
  int64_t forward_part, part_sum, forward_again, forward_bytes;
  int64_t delta, weight, ends, top, large, part, row_sums, part_bias, backward_again, backward_bytes;
};

inline int kernel_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : 128; }

inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }
inline int64_t room(int64_t floats) { return up(floats * 4, 256) * 256; }
// Takes room for `floats` at the end of a layout.
inline int64_t take(int64_t& end, int64_t floats) {
  const int64_t at = end;
  end += room(floats);
  return at;
}

// How many workgroups a panel's work is split over: enough to give every compute unit the `each` that it holds at a time, of at least
// `least` steps, and two of at least six if it holds one; if there are `from` steps, so that what is saved pays for the kernel that joins the
// parts.  (One at a time, us, 1 / 2 for each compute unit: fp32, 8 heads of 128 on one of 685 x 942, 15 tiles 41 / 54; 8 of 96 of 1277 x 294,
// training, 142 / 165; but 5 masked heads of 96 of 2627 x 2627, 41 tiles, 84 / 76, and fp16, 8 x 8 heads of 128 of 1188 x 1104 414 / 372.)
inline int split_count(int64_t blocks, int64_t steps, int each, int least, int from) {
  if (blocks <= 0 || steps < from) return 1;
  int64_t s = std::min<int64_t>(each * 256 / blocks, steps / least);
  if (each == 1) s = std::max(s, std::min<int64_t>(2 * 256 / blocks, steps / 6));
  return (int)std::min<int64_t>(std::max<int64_t>(s, 1), 64);
}

// backward: of the strides of dO, which the forward pass does not take, the plan of that is to know nothing
Plan make_plan(const spdl_attention_problem& p, int elem_bytes, bool backward) {
  Plan x{};
  const int64_t group = p.kv_heads ? p.heads / p.kv_heads : 1;
  x.rows = (int64_t)p.batch * p.heads * p.m;
  x.kv_rows = (int64_t)p.batch * p.kv_heads * p.k;
  x.width = kernel_width(p.d);
  x.token = p.m <= 16;
  // Tiles of 64 keys (or queries) per part at least, and from how many on a panel is split: a tile takes 2 to 4 us where a compute unit has one
  // workgroup, the kernel that joins the parts 4 (us, 1 / 2 / 4 tiles per part: fp32 training step of 3 x 6 heads of 77 x 203 85 / 95 / 117, fp16 one of
  // 2 heads of 22 x 1505 65 / 62 / 67; single tokens, 4 / 8 blocks of 32 keys: fp32 2 x 4 heads on 361 keys 18 / 26, fp16 7 x 14 rows on 3547 23 / 19).
  const bool f32 = elem_bytes == 4;
  const int least = f32 ? 1 : 2, from = f32 ? 3 : 6;
  const int each = x.width * (f32 ? 2 : 1) <= 128 ? 2 : 1;    // the launch bounds of the panel kernels
  if (x.token) {
    x.token_rows = group * p.m <= 4 ? 4 : !f32 ? 32 : group * p.m <= 8 ? 8 : 16;
    x.forward_blocks = (int64_t)p.batch * p.kv_heads * up(group * p.m, x.token_rows);
    x.forward_splits = split_count(x.forward_blocks, up(p.k, 32), 2, f32 ? 4 : 8, f32 ? 9 : 17);
  } else {
    x.forward_blocks = (int64_t)p.batch * p.heads * up(p.m, kAttnPanel);
    x.forward_splits = split_count(x.forward_blocks, up(p.k, kAttnTile), each, least, from);
  }
  x.dq_blocks = (int64_t)p.batch * p.heads * up(p.m, kAttnPanel);
  x.dq_splits = split_count(x.dq_blocks, up(p.k, kAttnTile), each, least, from);
  x.dkv_blocks = (int64_t)p.batch * p.kv_heads * up(p.k, kAttnPanel);
  x.dkv_splits = split_count(x.dkv_blocks, group * up(p.m, kAttnTile), x.width == 128 ? 1 : each, least, from);
  // tiles near the diagonal that a panel meets
  x.dbias_splits = split_count(x.dq_blocks, std::min<int64_t>(up(p.k, kAttnTile), (2 * p.span + kAttnPanel) / kAttnTile + 2), 2, 1, 3);
  x.parts = (int64_t)p.batch * up(p.m, kAttnPanel) * x.dbias_splits;
  // workgroups that look for the largest number of a head: of 64 rows at least, and no more of them in all than 2^16 for each operand
  const int64_t kv = std::max<int64_t>((int64_t)p.batch * p.kv_heads, 1);
  x.most_parts = (int)std::max<int64_t>(1, std::min<int64_t>({64, up(std::max<int64_t>(group * p.m, p.k), 64), (1 << 16) / kv}));

  int64_t terms = 0, end = 0;
  const int64_t longest = std::max({p.Q.row, p.K.row, p.V.row, backward ? p.dO.row : 0});
  x.copied = elem_bytes == 4 || p.d % 8 != 0 || longest >= 1 << 24;
  const int numbers = elem_bytes == 4 ? x.width : x.width / 2;    // floats' room that a row of terms takes
  if (x.copied) {
    x.most = take(terms, (int64_t)p.batch * p.kv_heads * 4 * x.most_parts);
    x.factors = take(terms, (int64_t)p.batch * p.kv_heads * 4);
    x.k16 = take(terms, x.kv_rows * numbers);
    x.v16 = take(terms, x.kv_rows * numbers);
    end = terms;
    x.q16 = take(terms, x.rows * numbers);
  }
  end = x.token ? 0 : elem_bytes == 4 ? end : terms;      // the forward pass in single precision needs no terms of Q
  if (x.forward_splits > 1) {
    x.forward_part = take(end, x.forward_splits * x.rows * p.d);
    x.part_sum = take(end, 2 * x.forward_splits * x.rows);
  }
  if (!x.token) x.forward_again = take(end, x.forward_blocks * x.forward_splits * kAttnWaves);
  x.forward_bytes = end;
  end = terms;
  if (x.copied) x.g16 = take(end, x.rows * numbers);
  x.delta = take(end, x.rows);
  x.weight = take(end, x.rows);
  x.ends = take(end, 2 * x.rows);
  x.top = take(end, x.rows);
  x.large = take(end, x.dq_blocks * kAttnWaves);
  x.part = take(end, std::max(x.dq_splits > 1 ? x.dq_splits * x.rows * p.d : 0, x.dkv_splits > 1 ? 2 * x.dkv_splits * x.kv_rows * p.d : 0));
  if (x.dq_splits > 1) x.row_sums = take(end, 2 * x.dq_splits * x.rows * kAttnRowSums);
  if (p.buckets > 0) {
    x.part_bias = take(end, x.parts * p.heads * (2 * (int64_t)p.span + 1));
  }
  x.backward_again = take(end, std::max(x.dq_blocks * x.dq_splits, x.dkv_blocks * x.dkv_splits) * kAttnWaves);
  x.backward_bytes = end;
  return x;
}

bool input_strides_ok(const spdl_strides& s) { return s.batch >= 0 && s.head >= 0 && s.row >= 0; }

// Whether no two elements of an output lie at one address: by ascending stride, each dimension steps over all of the ones below.
bool output_strides_ok(const spdl_strides& s, int64_t batch, int64_t heads, int64_t rows, int64_t d) {
  struct Dim { int64_t stride, size; } dims[3] = {{s.batch, batch}, {s.head, heads}, {s.row, rows}};
  std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  int64_t extent = d;
  for (const Dim& x : dims) {
    if (x.stride < 0) return false;
    if (x.size <= 1 || batch == 0 || heads == 0 || rows == 0) continue;
    if (x.stride < extent) return false;
    if (x.stride > (INT64_MAX / 8 - extent) / x.size) return false;
    extent += x.stride * (x.size - 1);
  }
  return true;
}

bool sizes_ok(const spdl_attention_problem& p) {
  if (p.batch < 0 || p.heads < 0 || p.kv_heads < 0 || p.m < 0 || p.k < 0 || p.d < 1 || p.m > kMostRows || p.k > kMostRows) return false;
  if ((p.heads == 0) != (p.kv_heads == 0) || (p.heads > 0 && p.heads % p.kv_heads)) return false;
  if (p.span < 0 || p.span > kAttnSpanMax || p.buckets < 0 || p.buckets > kAttnBucketsMax) return false;
  if (!std::isfinite(p.scale)) return false;
  // grids: of 256 threads to a workgroup, 2^32 in all; of single tokens there are at most heads (m / 4 + 1) workgroups to a sequence
  const int64_t bh = (int64_t)p.batch * p.heads;
  return bh <= (1 << 21) && bh * up(std::max(p.m, p.k), kAttnPanel) < (1 << 23);
}

int check(const spdl_attention_problem* p, const int* bucket_of, const void* table) {
  if (!p || !sizes_ok(*p)) return SPDL_ERR_INVALID;
  if (p->d > kMostWidth) return SPDL_ERR_UNSUPPORTED;
  if (!table != !bucket_of || (table && p->buckets < 1)) return SPDL_ERR_INVALID;
  if (!input_strides_ok(p->Q) || !input_strides_ok(p->K) || !input_strides_ok(p->V)) return SPDL_ERR_INVALID;
  return SPDL_OK;
}

AttnStrides strides(const spdl_strides& s) { return {s.batch, s.head, s.row}; }

AttnArgs make_args(const spdl_attention_problem& p, const void* Q, const void* K, const void* V, const int* lengths, const int* positions,
                   const void* mask, const int* bucket_of, const void* table, void* O, float* lse) {
  AttnArgs a{};
  a.batch = p.batch, a.heads = p.heads, a.kv_heads = p.kv_heads, a.group = p.kv_heads ? p.heads / p.kv_heads : 1;
  a.m = p.m, a.k = p.k, a.d = p.d, a.span = p.span, a.buckets = p.buckets, a.splits = 1, a.scale = p.scale;
  a.q = strides(p.Q), a.kk = strides(p.K), a.v = strides(p.V), a.o = strides(p.O);
  a.dout = strides(p.dO), a.dq = strides(p.dQ), a.dk = strides(p.dK), a.dv = strides(p.dV);
  a.Q = Q, a.K = K, a.V = V, a.lengths = lengths, a.positions = positions, a.bucket_of = bucket_of, a.table = table;
  a.mask = static_cast<const uint64_t*>(mask);
  a.O = O, a.lse = lse;
  return a;
}

bool launch(void (*kernel)(AttnArgs), int64_t blocks, int lds, AttnArgs a, hipStream_t stream) {
  a.by_length = a.lengths && a.batch > 1 && a.batch <= 64;
  if (lds > 64 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return false;
  kernel<<<dim3((unsigned)blocks), dim3(256), lds, stream>>>(a);
  return hipGetLastError() == hipSuccess;
}

// The operands as the panel kernels take them: the caller's arrays in half precision; in single precision their terms, made here.
template <typename T, int D>
bool prepare_operands(const Plan& x, AttnArgs& a, char* w, bool backward, hipStream_t stream) {
  if (!x.copied) {
    a.q16 = static_cast<const _Float16*>(a.Q), a.q16s = a.q;
    a.k16 = static_cast<const _Float16*>(a.K), a.k16s = a.kk;
    a.v16 = static_cast<const _Float16*>(a.V), a.v16s = a.v;
    a.g16 = static_cast<const _Float16*>(a.dO), a.g16s = a.dout;
    a.width = a.d;
    return true;
  }
  constexpr int kWidth = attn_terms<T>() * D;
  AttnOperands o{};
  auto operand = [&](const void* from, const AttnStrides& s, int64_t to, int group, int rows, int keys, const _Float16*& terms, AttnStrides& strides) {
    _Float16* at = reinterpret_cast<_Float16*>(w + to);
    o.of[o.count++] = {from, at, s, a.kv_heads, group, rows, keys};
    terms = at;
    strides = {(int64_t)a.kv_heads * group * rows * kWidth, (int64_t)rows * kWidth, kWidth};
  };
  const bool queries = backward || sizeof(T) == 2;        // (the forward kernel takes Q's numbers as they are)
  o.first = queries ? 0 : 1;
  if (queries) operand(a.Q, a.q, x.q16, a.group, a.m, 0, a.q16, a.q16s);
  operand(a.K, a.kk, x.k16, 1, a.k, 1, a.k16, a.k16s);
  operand(a.V, a.v, x.v16, 1, a.k, 1, a.v16, a.v16s);
  if (backward) operand(a.dO, a.dout, x.g16, a.group, a.m, 0, a.g16, a.g16s);
  a.width = kWidth;
  a.factors = reinterpret_cast<float*>(w + x.factors);
  o.batch = a.batch, o.kv_heads = a.kv_heads, o.d = a.d, o.k = a.k, o.parts = x.most_parts, o.lengths = a.lengths;
  o.most = reinterpret_cast<float*>(w + x.most), o.factors = reinterpret_cast<float*>(w + x.factors);
  const int64_t each = (int64_t)a.batch * a.kv_heads * o.count;
  // of few numbers the workgroups that make the terms find the largest themselves, which saves a launch
  const int64_t rows = std::max<int64_t>(queries ? (int64_t)a.group * a.m : 0, a.k);
  if (rows * a.d <= 32768) {
    o.most = nullptr;
  } else if (sizeof(T) == 4) {
    attention_largest_kernel<<<dim3((unsigned)(each * o.parts)), dim3(256), 0, stream>>>(o);
    if (hipGetLastError() != hipSuccess) return false;
  }
  if (rows == 0) return true;
  // (a grid holds fewer than 2^32 threads one way: the workgroups of a long operand take more than one block of rows)
  const int64_t blocks = up(rows, 256 / (D / 8));
  attention_terms_kernel<T, D><<<dim3((unsigned)std::min<int64_t>(blocks, 1 << 16), (unsigned)std::min<int64_t>(each, 32768)), dim3(256), 0, stream>>>(
      o, blocks, (int)each);
  return hipGetLastError() == hipSuccess;
}

template <typename T, int D, bool BIAS>
bool launch_forward(const Plan& x, AttnArgs a, char* w, hipStream_t stream) {
  if (x.token) {
    const int bias = BIAS ? std::min(a.group, x.token_rows) * a.buckets * 4 + (2 * a.span + 1) * 4 : 0;
    const int64_t blocks = x.forward_blocks * a.splits;
    if constexpr (sizeof(T) == 2) {
      // K and V of four waves, later their parts
      if (x.token_rows == 32) {
        const int lds = std::max(kAttnWaves * 2 * 32 * AttnTile<D, 1>::kPitch + bias, kAttnWaves * 32 * (D + 1 + 2) * 4);
        return launch(attention_tokens_kernel<D, BIAS>, blocks, lds, a, stream);
      }
    }
    constexpr int kColumns = 256 / sizeof(T);
    const int lds = std::max(bias, kAttnWaves * x.token_rows * ((D + kColumns - 1) / kColumns * kColumns + 4 + 2) * 4);
    if constexpr (sizeof(T) == 4) {
      if (x.token_rows == 8) return launch(attention_token_kernel<T, D, 8, BIAS>, blocks, lds, a, stream);
      if (x.token_rows == 16) return launch(attention_token_kernel<T, D, 16, BIAS>, blocks, lds, a, stream);
    }
    return launch(attention_token_kernel<T, D, 4, BIAS>, blocks, lds, a, stream);
  }
  if (!prepare_operands<T, D>(x, a, w, false, stream)) return false;
  using Tile = AttnTile<D, attn_terms<T>(), attn_queries_each<T, D>()>;
  const int lds = Tile::kSets * kAttnTile * (Tile::kPitch + Tile::kPitchT) + (BIAS ? attn_bias_entries(a.span, kAttnPad) * 4 : 0);
  a.again = reinterpret_cast<unsigned*>(w + x.forward_again);
  if (!launch(attention_forward_kernel<T, D, BIAS>, x.forward_blocks * a.splits, lds, a, stream)) return false;
  return !a.mask || launch(attention_forward_again_kernel<T>, x.forward_blocks * a.splits, 0, a, stream);
}

template <typename T, int D, bool BIAS>
bool launch_backward(const Plan& x, AttnArgs a, char* w, void* dtable, hipStream_t stream) {
  using Queries = AttnTile<D, attn_terms<T>(), attn_queries_each<T, D>()>;
  using Keys = AttnTile<D, attn_terms<T>(), attn_keys_each<T, D>()>;
  const int bias = BIAS ? attn_bias_entries(a.span, kAttnPadBlock) * 4 : 0;
  const int64_t pieces = up(a.d, 4);
  a.part = reinterpret_cast<float*>(w + x.part);
  a.again = reinterpret_cast<unsigned*>(w + x.backward_again);
  if ((x.dq_blocks > 0 || x.dkv_blocks > 0) && !prepare_operands<T, D>(x, a, w, true, stream)) return false;
  if (x.dq_blocks > 0) {
    a.splits = x.dq_splits;
    if (!launch(attention_dq_kernel<T, D, BIAS>, x.dq_blocks * a.splits, Queries::kSets * Queries::kPair + bias, a, stream)) return false;
    if (a.mask && !launch(attention_dq_again_kernel<T>, x.dq_blocks * a.splits, 0, a, stream)) return false;
    if (a.splits > 1) {
      attention_sum_dq_kernel<T, BIAS, attn_row_sums<T, BIAS>()><<<dim3((unsigned)up(x.rows * pieces, 256)), dim3(256), 0, stream>>>(a);
      if (hipGetLastError() != hipSuccess) return false;
    }
  }
  // dK and dV, and in the same launch the sums for the bias, unless the LDS that those take would leave fewer workgroups to a compute unit
  a.splits = x.dkv_splits, a.bias_splits = x.dbias_splits;
  const int64_t blocks = x.dkv_blocks * a.splits, bias_blocks = BIAS && a.part_bias ? x.dq_blocks * a.bias_splits : 0;
  const int lds = Keys::kSets * (Keys::kPair + 5 * kAttnTile * 4) + bias;
  const int bias_lds = Keys::kPair + bias + 16 + kAttnWaves * (kAttnDiagonalBlock + 2 * a.span + 1) * 4;
  const bool together = bias_blocks > 0 && std::max(lds, bias_lds) * attn_keys_each<T, D>() <= 160 * 1024;
  a.bias_from = (int)blocks;
  if (blocks + (together ? bias_blocks : 0) > 0 &&
      !launch(attention_dkv_kernel<T, D, BIAS>, blocks + (together ? bias_blocks : 0), together ? std::max(lds, bias_lds) : lds, a, stream))
    return false;
  if (bias_blocks > 0 && !together) {
    a.bias_from = 0;
    if (!launch(attention_dkv_kernel<T, D, BIAS>, bias_blocks, bias_lds, a, stream)) return false;
  }
  if (x.dkv_blocks > 0 && a.mask && !launch(attention_dkv_again_kernel<T>, x.dkv_blocks * a.splits, 0, a, stream)) return false;
  const int tables = dtable ? a.heads : 0, n = 2 * a.span + 1;
  const int64_t sums = a.splits > 1 ? up(2 * x.kv_rows * pieces, 1024) : 0;
  if (tables + sums == 0) return true;
  attention_finish_kernel<T><<<dim3((unsigned)(tables + sums)), dim3(1024), tables ? (n < 1024 ? 1024 / n : 1) * n * 8 + n * 4 : 0, stream>>>(
      a, tables, (int)x.parts, static_cast<T*>(dtable));
  return hipGetLastError() == hipSuccess;
}

template <typename T, bool BIAS>
bool dispatch_forward(const Plan& x, const AttnArgs& a, char* w, hipStream_t stream) {
  if (a.d <= 32) return launch_forward<T, 32, BIAS>(x, a, w, stream);
  if (a.d <= 64) return launch_forward<T, 64, BIAS>(x, a, w, stream);
  if (a.d <= 96) return launch_forward<T, 96, BIAS>(x, a, w, stream);
  return launch_forward<T, 128, BIAS>(x, a, w, stream);
}

template <typename T, bool BIAS>
bool dispatch_backward(const Plan& x, const AttnArgs& a, char* w, void* dtable, hipStream_t stream) {
  if (a.d <= 32) return launch_backward<T, 32, BIAS>(x, a, w, dtable, stream);
  if (a.d <= 64) return launch_backward<T, 64, BIAS>(x, a, w, dtable, stream);
  if (a.d <= 96) return launch_backward<T, 96, BIAS>(x, a, w, dtable, stream);
  return launch_backward<T, 128, BIAS>(x, a, w, dtable, stream);
}

inline bool workspace_ok(const void* workspace, int64_t bytes, int64_t needed) {
  return needed == 0 || (workspace && bytes >= needed && reinterpret_cast<uintptr_t>(workspace) % 16 == 0);
}

template <typename T>
int attention(const spdl_attention_problem* p, const void* Q, const void* K, const void* V, const int* lengths, const int* positions,
              const void* mask, const int* bucket_of, const void* table, void* O, float* lse, void* workspace, int64_t workspace_bytes,
              void* stream) {
  const int bad = check(p, bucket_of, table);
  if (bad != SPDL_OK) return bad;
  if (!output_strides_ok(p->O, p->batch, p->heads, p->m, p->d)) return SPDL_ERR_INVALID;
  if (p->batch == 0 || p->heads == 0 || p->m == 0) return SPDL_OK;
  if (!Q || !O || (p->k > 0 && (!K || !V))) return SPDL_ERR_INVALID;
  const Plan x = make_plan(*p, sizeof(T), false);
  if (!workspace_ok(workspace, workspace_bytes, x.forward_bytes)) return SPDL_ERR_INVALID;
  AttnArgs a = make_args(*p, Q, K, V, lengths, positions, mask, bucket_of, table, O, lse);
  a.splits = x.forward_splits;
  char* w = static_cast<char*>(workspace);
  a.part = reinterpret_cast<float*>(w + x.forward_part);
  a.part_sum = reinterpret_cast<float2*>(w + x.part_sum);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (!(table ? dispatch_forward<T, true>(x, a, w, s) : dispatch_forward<T, false>(x, a, w, s))) return SPDL_ERR_LAUNCH;
  if (a.splits > 1) {
    if (x.rows >= 4096 && a.splits <= 16)
      attention_join_kernel<T, 16><<<dim3((unsigned)up(x.rows, 16)), dim3(256), 0, s>>>(a);
    else
      attention_join_kernel<T, 64><<<dim3((unsigned)up(x.rows, 4)), dim3(256), 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return SPDL_ERR_LAUNCH;
  }
  return SPDL_OK;
}

template <typename T>
int attention_backward(const spdl_attention_problem* p, const void* Q, const void* K, const void* V, const int* lengths, const int* positions,
                       const void* mask, const int* bucket_of, const void* table, const void* O, const float* lse, const void* dO, void* dQ,
                       void* dK, void* dV, void* dtable, void* workspace, int64_t workspace_bytes, void* stream) {
  const int bad = check(p, bucket_of, table);
  if (bad != SPDL_OK) return bad;
  if (dtable && !table) return SPDL_ERR_INVALID;
  if (!input_strides_ok(p->O) || !input_strides_ok(p->dO)) return SPDL_ERR_INVALID;
  if (!output_strides_ok(p->dQ, p->batch, p->heads, p->m, p->d) || !output_strides_ok(p->dK, p->batch, p->kv_heads, p->k, p->d) ||
      !output_strides_ok(p->dV, p->batch, p->kv_heads, p->k, p->d))
    return SPDL_ERR_INVALID;
  if (p->heads == 0) return SPDL_OK;
  const bool queries = p->batch > 0 && p->m > 0, keys = p->batch > 0 && p->k > 0;
  if (queries && (!Q || !O || !lse || !dO || !dQ)) return SPDL_ERR_INVALID;
  if (keys && (!K || !V || !dK || !dV)) return SPDL_ERR_INVALID;
  const Plan x = make_plan(*p, sizeof(T), true);
  if ((queries || keys) && !workspace_ok(workspace, workspace_bytes, x.backward_bytes)) return SPDL_ERR_INVALID;
  AttnArgs a = make_args(*p, Q, K, V, lengths, positions, mask, bucket_of, table, const_cast<void*>(O), const_cast<float*>(lse));
  a.dO = dO, a.dQ = dQ, a.dK = dK, a.dV = dV;
  char* w = static_cast<char*>(workspace);
  a.delta = reinterpret_cast<float*>(w + x.delta);
  a.weight = reinterpret_cast<float*>(w + x.weight);
  a.ends = reinterpret_cast<float*>(w + x.ends);
  a.top = reinterpret_cast<float*>(w + x.top);
  a.large = reinterpret_cast<int*>(w + x.large);
  a.row_sums = reinterpret_cast<double*>(w + x.row_sums);
  a.part_bias = dtable ? reinterpret_cast<float*>(w + x.part_bias) : nullptr;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (!(table ? dispatch_backward<T, true>(x, a, w, dtable, s) : dispatch_backward<T, false>(x, a, w, dtable, s))) return SPDL_ERR_LAUNCH;
  return SPDL_OK;
}

}  // namespace

extern "C" {

int64_t spdl_attention_workspace(const spdl_attention_problem* p, int elem_bytes, int backward) {
  if (!p || !sizes_ok(*p) || p->d > kMostWidth || (elem_bytes != 2 && elem_bytes != 4)) return SPDL_ERR_INVALID;
  const int64_t forward = make_plan(*p, elem_bytes, false).forward_bytes;
  return backward ? std::max(forward, make_plan(*p, elem_bytes, true).backward_bytes) : forward;
}

int spdl_attention(const spdl_attention_problem* problem, const float* Q, const float* K, const float* V, const int* lengths,
                   const int* positions, const void* mask, const int* bucket_of, const float* table, float* O, float* lse, void* workspace,
                   int64_t workspace_bytes, void* stream) {
  return attention<float>(problem, Q, K, V, lengths, positions, mask, bucket_of, table, O, lse, workspace, workspace_bytes, stream);
}
int spdl_attention_f16(const spdl_attention_problem* problem, const uint16_t* Q, const uint16_t* K, const uint16_t* V, const int* lengths,
                       const int* positions, const void* mask, const int* bucket_of, const uint16_t* table, uint16_t* O, float* lse,
                       void* workspace, int64_t workspace_bytes, void* stream) {
  return attention<_Float16>(problem, Q, K, V, lengths, positions, mask, bucket_of, table, O, lse, workspace, workspace_bytes, stream);
}

int spdl_attention_backward(const spdl_attention_problem* problem, const float* Q, const float* K, const float* V, const int* lengths,
                            const int* positions, const void* mask, const int* bucket_of, const float* table, const float* O,
                            const float* lse, const float* dO, float* dQ, float* dK, float* dV, float* dtable, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  return attention_backward<float>(problem, Q, K, V, lengths, positions, mask, bucket_of, table, O, lse, dO, dQ, dK, dV, dtable, workspace,
                                   workspace_bytes, stream);
}
int spdl_attention_backward_f16(const spdl_attention_problem* problem, const uint16_t* Q, const uint16_t* K, const uint16_t* V,
                                const int* lengths, const int* positions, const void* mask, const int* bucket_of, const uint16_t* table,
                                const uint16_t* O, const float* lse, const uint16_t* dO, uint16_t* dQ, uint16_t* dK, uint16_t* dV,
                                uint16_t* dtable, void* workspace, int64_t workspace_bytes, void* stream) {
  return attention_backward<_Float16>(problem, Q, K, V, lengths, positions, mask, bucket_of, table, O, lse, dO, dQ, dK, dV, dtable, workspace,
                                      workspace_bytes, stream);
}

int64_t spdl_attention_mask_bytes(int m, int k) {
  if (m < 0 || k < 0 || m > kMostRows || k > kMostRows) return SPDL_ERR_INVALID;
  return MaskLayout(m, k).words * 8;
}

int spdl_build_attention_mask(int m, int k, int nnz, const int* row_offsets, const int* column_indices, void* mask, void* stream) {
  if (m < 0 || k < 0 || nnz < 0 || m > kMostRows || k > kMostRows) return SPDL_ERR_INVALID;
  const MaskLayout lay(m, k);
  if (lay.words == 0) return SPDL_OK;
  if (!mask || reinterpret_cast<uintptr_t>(mask) % 8 || (nnz > 0 && (!row_offsets || !column_indices))) return SPDL_ERR_INVALID;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  auto* bits = static_cast<uint64_t*>(mask);
  const auto grid = [](int64_t blocks) { return dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)); };   // whose workgroups take more than one
  const int64_t clear_from = nnz == 0 ? 0 : lay.row_tiles;    // the words are written whole
  attention_mask_clear_kernel<<<grid(up(lay.words - clear_from, 256)), dim3(256), 0, s>>>(lay.words - clear_from, bits + clear_from);
  if (hipGetLastError() != hipSuccess) return SPDL_ERR_LAUNCH;
  if (nnz == 0) return SPDL_OK;
  auto rows = [&](auto kernel, int64_t each) {
    const int64_t words = std::min(lay.tj, kMaskWords / each);
    kernel<<<grid(lay.ti * (64 / each) * up(lay.tj, words)), dim3(256), words * each * 8, s>>>(m, k, row_offsets, column_indices, bits);
  };
  if (lay.tj * 16 <= kMaskWords) rows(attention_mask_rows_kernel<16>, 16);
  else if (lay.tj * 4 <= kMaskWords) rows(attention_mask_rows_kernel<4>, 4);
  else rows(attention_mask_rows_kernel<1>, 1);
  if (hipGetLastError() != hipSuccess) return SPDL_ERR_LAUNCH;
  attention_mask_tiles_kernel<<<grid(up(lay.ti * lay.tj, 4)), dim3(256), 0, s>>>(m, k, bits);
  return hipGetLastError() == hipSuccess ? SPDL_OK : SPDL_ERR_LAUNCH;
}

int spdl_build_relative_buckets_host(int buckets, int max_distance, int bidirectional, int* bucket_of) {
  if (!bucket_of || buckets < 1 || buckets > kAttnBucketsMax || max_distance < 1 || max_distance > kAttnSpanMax) return SPDL_ERR_INVALID;
  const int side = bidirectional ? buckets / 2 : buckets, exact = side / 2, steps = side - exact;
  if (exact < 1 || max_distance <= exact) return SPDL_ERR_INVALID;
  for (int rel = -max_distance; rel <= max_distance; ++rel) {
    const int n = bidirectional ? std::abs(rel) : std::max(-rel, 0);
    int b = n;
    if (n >= exact) {
      // the most e with (n / exact)^steps >= (max_distance / exact)^e; the two sides are equal or far more than 1e-12 apart
      const double x = steps * std::log((double)n / exact) / std::log((double)max_distance / exact);
      b = exact + std::min(steps - 1, (int)std::floor(x + 1e-11));
    }
    bucket_of[rel + max_distance] = b + (bidirectional && rel > 0 ? side : 0);
  }
  return SPDL_OK;
}

}  // extern "C"
