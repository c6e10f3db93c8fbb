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
  bool token;                          // the kernel for a few queries
  int forward_splits, dq_splits, dkv_splits;
  int64_t forward_blocks, dq_blocks, dkv_blocks;      // without the splits
  int64_t rows, kv_rows, parts;        // parts: workgroups that leave sums of dS per head
  // offsets into the workspace, in bytes
  int64_t part_lse, forward_bytes;
  int64_t delta, part, part_bias, backward_bytes;
};

inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }
inline int64_t room(int64_t floats) { return up(floats * 4, 256) * 256; }

// How many workgroups a panel's work is split over: enough to give every compute unit `want` of them, of at least `least` steps each.
inline int split_count(int64_t blocks, int64_t steps, int want, int least) {
  if (blocks <= 0 || steps <= 0) return 1;
  const int64_t s = std::min<int64_t>(want * 256 / blocks, steps / least);
  return (int)std::min<int64_t>(std::max<int64_t>(s, 1), 64);
}

Plan make_plan(const spdl_attention_problem& p) {
  Plan x{};
  const int64_t group = p.kv_heads ? p.heads / p.kv_heads : 1;
  x.rows = (int64_t)p.batch * p.heads * p.m;
  x.kv_rows = (int64_t)p.batch * p.kv_heads * p.k;
  x.token = p.m <= 16;
  if (x.token) {
    x.forward_blocks = (int64_t)p.batch * p.kv_heads * up(group * p.m, 32);
    x.forward_splits = split_count(x.forward_blocks, up(p.k, 32), 4, 8);
  } else {
    x.forward_blocks = (int64_t)p.batch * p.heads * up(p.m, kAttnPanel);
    x.forward_splits = split_count(x.forward_blocks, up(p.k, kAttnTile), 2, 4);
  }
  x.dq_blocks = (int64_t)p.batch * p.heads * up(p.m, kAttnPanel);
  x.dq_splits = split_count(x.dq_blocks, up(p.k, kAttnTile), 2, 4);
  x.dkv_blocks = (int64_t)p.batch * p.kv_heads * up(p.k, kAttnPanel);
  x.dkv_splits = split_count(x.dkv_blocks, group * up(p.m, kAttnTile), 2, 4);
  x.part_lse = x.forward_splits > 1 ? room(x.forward_splits * x.rows * p.d) : 0;
  x.forward_bytes = x.forward_splits > 1 ? x.part_lse + room(x.forward_splits * x.rows) : 0;
  x.parts = (int64_t)p.batch * up(p.m, kAttnPanel) * x.dq_splits;
  x.delta = 0;
  x.part = room(x.rows);
  x.part_bias = x.part + room(std::max(x.dq_splits > 1 ? x.dq_splits * x.rows * p.d : 0, x.dkv_splits > 1 ? 2 * x.dkv_splits * x.kv_rows * p.d : 0));
  x.backward_bytes = x.part_bias + (p.buckets > 0 ? room(x.parts * p.heads * (2 * (int64_t)p.span + 1)) : 0);
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
  if (p.heads > 0 && (p.kv_heads < 1 || p.heads % p.kv_heads)) return false;
  if (p.span < 0 || p.span > kAttnSpanMax || p.buckets < 0 || p.buckets > kAttnBucketsMax) return false;
  if (!std::isfinite(p.scale)) return false;
  // grids, and sizes of the workspace
  const int64_t bh = (int64_t)p.batch * p.heads;
  return bh < (1 << 24) && bh * std::max(p.m, 1) < ((int64_t)1 << 36) && bh * std::max(p.k, 1) < ((int64_t)1 << 36) &&
         bh * up(std::max(p.m, p.k), 32) < ((int64_t)1 << 30);
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

bool launch(void (*kernel)(AttnArgs), int64_t blocks, int lds, const AttnArgs& a, hipStream_t stream) {
  if (lds > 64 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return false;
  kernel<<<dim3((unsigned)blocks), dim3(256), lds, stream>>>(a);
  return hipGetLastError() == hipSuccess;
}

template <typename T, int D, bool BIAS>
bool launch_forward(const Plan& x, const AttnArgs& a, hipStream_t stream) {
  constexpr int kPitch = AttnTile<T, D>::kPitch;
  if (x.token) {
    const int lds = kAttnWaves * 2 * 32 * kPitch + (BIAS ? std::min(a.group, 32) * a.buckets * 4 + (2 * a.span + 1) * 4 : 0);
    return launch(attention_token_kernel<T, D, BIAS>, x.forward_blocks * a.splits, lds, a, stream);
  }
  const int lds = 2 * kAttnTile * kPitch + (BIAS ? attn_bias_entries(a.span) * 4 : 0);
  return launch(attention_forward_kernel<T, D, BIAS>, x.forward_blocks * a.splits, lds, a, stream);
}

template <typename T, int D, bool BIAS>
bool launch_backward(const Plan& x, AttnArgs a, float* part, hipStream_t stream) {
  constexpr int kTiles = 2 * kAttnTile * AttnTile<T, D>::kPitch;
  a.part = part;
  const int64_t vec = (int64_t)a.d;
  if (x.dq_blocks > 0) {
    a.splits = x.dq_splits;
    const int lds = kTiles + (BIAS ? attn_bias_entries(a.span) * 4 : 0) +
                    (BIAS && a.part_bias ? kAttnWaves * (kAttnDiagBytes + (2 * a.span + 1) * 4) : 0);
    if (!launch(attention_dq_kernel<T, D, BIAS>, x.dq_blocks * a.splits, lds, a, stream)) return false;
    if (a.splits > 1) {
      attention_sum_kernel<T><<<dim3((unsigned)up(x.rows * vec, 256)), dim3(256), 0, stream>>>(a.splits, x.rows, a.heads, a.m, a.d, part, a.dq,
                                                                                              static_cast<T*>(a.dQ));
      if (hipGetLastError() != hipSuccess) return false;
    }
  }
  if (x.dkv_blocks > 0) {
    a.splits = x.dkv_splits;
    const int lds = kTiles + 2 * kAttnTile * 4 + (BIAS ? attn_bias_entries(a.span) * 4 : 0);
    if (!launch(attention_dkv_kernel<T, D, BIAS>, x.dkv_blocks * a.splits, lds, a, stream)) return false;
    for (int which = 0; which < 2 && a.splits > 1; ++which) {
      attention_sum_kernel<T><<<dim3((unsigned)up(x.kv_rows * vec, 256)), dim3(256), 0, stream>>>(
          a.splits, x.kv_rows, a.kv_heads, a.k, a.d, part + which * a.splits * x.kv_rows * vec, which ? a.dv : a.dk,
          static_cast<T*>(which ? a.dV : a.dK));
      if (hipGetLastError() != hipSuccess) return false;
    }
  }
  return true;
}

template <typename T, bool BIAS>
bool dispatch_forward(const Plan& x, const AttnArgs& a, hipStream_t stream) {
  if (a.d <= 32) return launch_forward<T, 32, BIAS>(x, a, stream);
  if (a.d <= 64) return launch_forward<T, 64, BIAS>(x, a, stream);
  if (a.d <= 96) return launch_forward<T, 96, BIAS>(x, a, stream);
  return launch_forward<T, 128, BIAS>(x, a, stream);
}

template <typename T, bool BIAS>
bool dispatch_backward(const Plan& x, const AttnArgs& a, float* part, hipStream_t stream) {
  if (a.d <= 32) return launch_backward<T, 32, BIAS>(x, a, part, stream);
  if (a.d <= 64) return launch_backward<T, 64, BIAS>(x, a, part, stream);
  if (a.d <= 96) return launch_backward<T, 96, BIAS>(x, a, part, stream);
  return launch_backward<T, 128, BIAS>(x, a, part, stream);
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
  const Plan x = make_plan(*p);
  if (!workspace_ok(workspace, workspace_bytes, x.forward_bytes)) return SPDL_ERR_INVALID;
  AttnArgs a = make_args(*p, Q, K, V, lengths, positions, mask, bucket_of, table, O, lse);
  a.splits = x.forward_splits;
  a.part = static_cast<float*>(workspace);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + x.part_lse);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (!(table ? dispatch_forward<T, true>(x, a, s) : dispatch_forward<T, false>(x, a, s))) return SPDL_ERR_LAUNCH;
  if (a.splits > 1) {
    attention_join_kernel<T><<<dim3((unsigned)up(x.rows, 4)), dim3(256), 0, s>>>(a);
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
  const Plan x = make_plan(*p);
  if ((queries || keys) && !workspace_ok(workspace, workspace_bytes, x.backward_bytes)) return SPDL_ERR_INVALID;
  AttnArgs a = make_args(*p, Q, K, V, lengths, positions, mask, bucket_of, table, const_cast<void*>(O), const_cast<float*>(lse));
  a.dO = dO, a.dQ = dQ, a.dK = dK, a.dV = dV;
  char* w = static_cast<char*>(workspace);
  a.delta = reinterpret_cast<float*>(w + x.delta);
  a.part_bias = dtable ? reinterpret_cast<float*>(w + x.part_bias) : nullptr;
  float* part = reinterpret_cast<float*>(w + x.part);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (!(table ? dispatch_backward<T, true>(x, a, part, s) : dispatch_backward<T, false>(x, a, part, s))) return SPDL_ERR_LAUNCH;
  if (dtable) {
    attention_dtable_kernel<T><<<dim3((unsigned)p->heads), dim3(1024), (2 * p->span + 1) * 4, s>>>(a, (int)x.parts, static_cast<T*>(dtable));
    if (hipGetLastError() != hipSuccess) return SPDL_ERR_LAUNCH;
  }
  return SPDL_OK;
}

}  // namespace

extern "C" {

int64_t spdl_attention_workspace(const spdl_attention_problem* p, int elem_bytes, int backward) {
  if (!p || !sizes_ok(*p) || p->d > kMostWidth || (elem_bytes != 2 && elem_bytes != 4)) return SPDL_ERR_INVALID;
  const Plan x = make_plan(*p);
  return backward ? std::max(x.forward_bytes, x.backward_bytes) : x.forward_bytes;
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
  const int64_t words = MaskLayout(m, k).words;
  if (words == 0) return SPDL_OK;
  if (!mask || reinterpret_cast<uintptr_t>(mask) % 8 || (nnz > 0 && (!row_offsets || !column_indices))) return SPDL_ERR_INVALID;
  if (up(words, 256) > INT32_MAX) return SPDL_ERR_INVALID;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  attention_mask_clear_kernel<<<dim3((unsigned)up(words, 256)), dim3(256), 0, s>>>(words, static_cast<uint64_t*>(mask));
  if (hipGetLastError() != hipSuccess) return SPDL_ERR_LAUNCH;
  if (nnz == 0) return SPDL_OK;
  attention_mask_kernel<<<dim3((unsigned)up(m, 4)), dim3(256), 0, s>>>(m, k, row_offsets, column_indices, static_cast<unsigned long long*>(mask));
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
