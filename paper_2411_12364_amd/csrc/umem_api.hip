// The C ABI of libumem: argument validation, workspace layout and kernel sequencing.
// Every entry point validates everything before it enqueues anything.
#include <stdint.h>

#include <cmath>

#include <algorithm>
#include <mutex>

#include "umem_internal.h"

using namespace umem;

namespace {

constexpr size_t kAlign = 256;

size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int64_t isqrt64(int64_t x) {
  int64_t r = 0;
  while ((r + 1) * (r + 1) <= x) ++r;
  return r;
}

umem_status check_desc(const umem_desc* d) {
  if (d == nullptr) return UMEM_ERR_INVALID_ARG;
  if (d->heads < 1 || d->dk < 1 || d->n_keys < 1 || d->rank < 1 || d->topk < 1 || d->topm < 1 ||
      d->dv < 1 || d->expand < 1 || d->n_values < 1 || d->dv_virt < 0 || d->d_out < 0)
    return UMEM_ERR_INVALID_ARG;
  if (d->grid != UMEM_GRID_ADD && d->grid != UMEM_GRID_TUCKER) return UMEM_ERR_INVALID_ARG;
  if (d->weight != UMEM_W_RAW && d->weight != UMEM_W_SOFTMAX) return UMEM_ERR_INVALID_ARG;
  if (d->vdtype != UMEM_F32 && d->vdtype != UMEM_BF16) return UMEM_ERR_INVALID_ARG;
  if (d->cores < 0) return UMEM_ERR_INVALID_ARG;
  if (d->cores > 1) {
    if (d->grid != UMEM_GRID_TUCKER || d->weight != UMEM_W_RAW || d->dv % d->cores != 0)
      return UMEM_ERR_INVALID_ARG;
    if (!cores_supported(d->dv, d->vdtype, d->cores)) return UMEM_ERR_UNSUPPORTED;
  }
  if (d->dk % d->rank != 0) return UMEM_ERR_INVALID_ARG;
  if (d->grid == UMEM_GRID_ADD && d->rank != 1) return UMEM_ERR_INVALID_ARG;
  if (d->topk > d->n_keys) return UMEM_ERR_INVALID_ARG;
  if (static_cast<int64_t>(d->topm) > static_cast<int64_t>(d->topk) * d->topk)
    return UMEM_ERR_INVALID_ARG;
  const int64_t e = isqrt64(d->expand);
  if (e * e != d->expand) return UMEM_ERR_INVALID_ARG;
  if (d->expand > 1 && d->dv_virt == 0) return UMEM_ERR_INVALID_ARG;
  if (d->n_keys > kMaxSelect) return UMEM_ERR_UNSUPPORTED;   // also keeps n*n < 2^31
  if (static_cast<int64_t>(d->n_keys) * d->n_keys != d->n_values * d->expand)
    return UMEM_ERR_INVALID_ARG;
  if (d->topk > kMaxTopK || d->topk * d->topk > kMaxSelect || d->topm > kMaxTopM)
    return UMEM_ERR_UNSUPPORTED;
  if (d->grid == UMEM_GRID_TUCKER && d->topk > kMaxTopKTucker) return UMEM_ERR_UNSUPPORTED;
  if (d->grid == UMEM_GRID_ADD && additive_candidates(d->topk, d->topm) > 2048) return UMEM_ERR_UNSUPPORTED;
  if (d->rank > kMaxRank || (d->dk / d->rank) % 4 != 0 || d->dk > kMaxDk) return UMEM_ERR_UNSUPPORTED;
  if (d->heads > kMaxHeads || d->heads * d->topm > kMaxBag) return UMEM_ERR_UNSUPPORTED;
  if (d->expand > kMaxExpand) return UMEM_ERR_UNSUPPORTED;
  if (!gather_row_supported(d->dv, d->vdtype)) return UMEM_ERR_UNSUPPORTED;
  if (d->dv_virt % 8 != 0 || d->d_out % 8 != 0) return UMEM_ERR_UNSUPPORTED;   // 16-byte weight rows
  if (d->dv_virt > 0 && ((static_cast<int64_t>(d->expand) * d->dv) % 8 != 0 ||
                         !gemm_weight_supported(d->dv_virt, static_cast<int64_t>(d->expand) * d->dv) ||
                         !gemm_weight_supported(d->d_out, d->dv_virt)))
    return UMEM_ERR_UNSUPPORTED;
  // the output linear alone reads the pooled rows (bf16) in 16-byte pieces of 8
  if (d->dv_virt == 0 && d->d_out > 0 && (d->dv % 8 != 0 || !gemm_weight_supported(d->d_out, d->dv)))
    return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

umem_status check_tokens(int32_t T) {
  if (T < 0) return UMEM_ERR_INVALID_ARG;
  if (T > kMaxTokens) return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

umem_status check_scoring_ptrs(const umem_desc* d, const float* q_row, const float* q_col,
                               const float* k_row, const float* k_col, const float* core) {
  if (!q_row || !q_col || !k_row || !k_col) return UMEM_ERR_INVALID_ARG;
  if (!aligned(q_row, 16) || !aligned(q_col, 16) || !aligned(k_row, 16) || !aligned(k_col, 16))
    return UMEM_ERR_INVALID_ARG;
  if (d->grid == UMEM_GRID_TUCKER && (core == nullptr || !aligned(core, 4))) return UMEM_ERR_INVALID_ARG;
  return UMEM_OK;
}

struct Layout {
  size_t factors, sel, idx, w, pooled, proj, total;
};

// Workspace: [rank-1 factors (Tucker)] [selection scores] [idx] [w] [pooled, bf16] [projection
// scratch: the intermediate and split-K partials; before the projection, the scoring's fp16
// planes of queries and keys, dead once the scores are written]
Layout layout(const umem_desc* d, int32_t T) {
  Layout L{};
  const size_t th = static_cast<size_t>(T) * d->heads;
  size_t off = 0;
  L.factors = off;
  if (d->grid == UMEM_GRID_TUCKER) off += round_up(kFactorBytes);
  L.sel = off;
  off += round_up(2 * th * d->n_keys * sizeof(float));
  L.idx = off;
  off += round_up(th * d->topm * sizeof(int32_t));
  L.w = off;
  off += round_up(th * d->topm * n_cores(*d) * sizeof(float));
  L.pooled = off;
  if (d->dv_virt > 0 || d->d_out > 0)
    off += round_up(static_cast<size_t>(T) * d->expand * d->dv * sizeof(uint16_t));
  L.proj = off;
  const size_t proj = (d->dv_virt > 0 || d->d_out > 0)
                          ? project_workspace_bytes(T, d->expand, d->dv, d->dv_virt, d->d_out) : 0;
  off += round_up(std::max(proj, score_planes_bytes(*d, T)));
  L.total = off;
  return L;
}

// The most bytes that T tokens or fewer take, so that a workspace sized once for the longest batch does for the
// shorter ones.  A product over a long K is split in more ways where it has fewer tiles, and its partial sums
// can then take more (a query of 2,048 by 896: 576 tokens 20.9 MB, 577 12.7).  The split changes at tiles of 64
// rows alone, and between them every part grows.  A call itself asks for no more than it takes.
template <typename F>
size_t most_upto(int64_t T, F bytes) {
  size_t most = bytes(static_cast<int32_t>(T));
  for (int64_t t = 64; t < T; t += 64) most = std::max(most, bytes(static_cast<int32_t>(t)));
  return most;
}

umem_status check_ws(const umem_desc* d, int32_t T, const void* ws, size_t ws_bytes) {
  const Layout L = layout(d, T);
  if (L.total > 0 && (ws == nullptr || !aligned(ws, kAlign) || ws_bytes < L.total))
    return UMEM_ERR_WORKSPACE;
  return UMEM_OK;
}

umem_status hip_status(hipError_t e) { return e == hipSuccess ? UMEM_OK : UMEM_ERR_HIP; }

umem_status check_gather(int64_t n_values, int32_t dv, int32_t vdtype, const void* values,
                         int32_t T, int32_t bag, const int32_t* idx, const float* w,
                         int32_t expand, int32_t cores, const float* out) {
  if (n_values < 1 || dv < 1 || bag < 1 || expand < 1 || cores < 0) return UMEM_ERR_INVALID_ARG;
  if (cores > 1 && dv % cores != 0) return UMEM_ERR_INVALID_ARG;
  if (vdtype != UMEM_F32 && vdtype != UMEM_BF16) return UMEM_ERR_INVALID_ARG;
  umem_status st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!values || !idx || !w || !out) return UMEM_ERR_INVALID_ARG;
  if (!aligned(values, 16) || !aligned(out, 16) || !aligned(idx, 4) || !aligned(w, 4))
    return UMEM_ERR_INVALID_ARG;
  const int64_t esize = vdtype == UMEM_F32 ? 4 : 2;
  if (n_values > (INT64_C(1) << 62) / (static_cast<int64_t>(dv) * esize)) return UMEM_ERR_INVALID_ARG;
  if (n_values * expand > (INT64_C(1) << 31)) return UMEM_ERR_UNSUPPORTED;
  if (bag > kMaxBag || expand > kMaxExpand) return UMEM_ERR_UNSUPPORTED;
  if (!gather_row_supported(dv, vdtype)) return UMEM_ERR_UNSUPPORTED;
  if (cores > 1 && !cores_supported(dv, vdtype, cores)) return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

// The shape of a projection: w_proj given iff dv_virt > 0 (else the output linear alone, which
// needs expand == 1 and d_out > 0); w_out given iff d_out > 0.
umem_status check_project_shape(int32_t expand, int32_t dv, int32_t dv_virt, int32_t d_out,
                                bool has_proj, bool has_out) {
  if (expand < 1 || dv < 1 || dv_virt < 0 || d_out < 0) return UMEM_ERR_INVALID_ARG;
  if (has_proj != (dv_virt > 0) || has_out != (d_out > 0)) return UMEM_ERR_INVALID_ARG;
  if (!has_proj && (expand != 1 || d_out == 0)) return UMEM_ERR_INVALID_ARG;
  // the GEMMs read 16-byte pieces of rows of K: 4 fp32 of a pooled row, 8 bf16 of a weight row
  const int64_t k1 = static_cast<int64_t>(expand) * dv;
  if (k1 % 8 != 0 || dv_virt % 8 != 0 || d_out % 8 != 0) return UMEM_ERR_UNSUPPORTED;
  if (has_proj ? !gemm_weight_supported(dv_virt, k1) || (has_out && !gemm_weight_supported(d_out, dv_virt))
               : !gemm_weight_supported(d_out, dv))
    return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

umem_status check_project(int32_t T, int32_t expand, int32_t dv, int32_t dv_virt, int32_t d_out,
                          const float* pooled, const uint16_t* w_proj, const uint16_t* w_out,
                          const float* out, const void* ws, size_t ws_bytes) {
  umem_status st = check_project_shape(expand, dv, dv_virt, d_out, w_proj != nullptr, w_out != nullptr);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!pooled || !out) return UMEM_ERR_INVALID_ARG;
  const size_t need = project_workspace_bytes(T, expand, dv, dv_virt, d_out);
  if (need > 0 && (ws == nullptr || !aligned(ws, 16) || ws_bytes < need)) return UMEM_ERR_WORKSPACE;
  if (!aligned(pooled, 16) || !aligned(w_proj, 16) || !aligned(w_out, 16)) return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

hipError_t run_project(int32_t T, int32_t expand, int32_t dv, int32_t dv_virt, int32_t d_out,
                       const float* pooled, const uint16_t* w_proj, const uint16_t* w_out,
                       float* out, void* ws, hipStream_t s) {
  return launch_project(T, expand, dv, dv_virt, d_out, pooled, w_proj, w_out, out, ws, s);
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_workspace_size(const umem_desc* desc, int32_t T, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  const bool project = desc->dv_virt > 0 || desc->d_out > 0;
  *bytes = project ? most_upto(T, [=](int32_t t) { return layout(desc, t).total; }) : layout(desc, T).total;
  return UMEM_OK;
}

UMEM_API umem_status umem_axis_scores(const umem_desc* desc, int32_t T, const float* q_row,
                                      const float* q_col, const float* k_row, const float* k_col,
                                      const float* core, float* sel, void* ws, size_t ws_bytes,
                                      hipStream_t stream) {
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (st == UMEM_OK) st = check_scoring_ptrs(desc, q_row, q_col, k_row, k_col, core);
  if (st == UMEM_OK && (sel == nullptr || !aligned(sel, 4))) st = UMEM_ERR_INVALID_ARG;
  const bool tucker = desc->grid == UMEM_GRID_TUCKER;
  // [factors (Tucker)] [fp16 planes of the many-token path]
  const size_t planes_at = tucker ? round_up(kFactorBytes) : 0;
  const size_t planes = score_planes_bytes(*desc, T);
  const size_t need = planes > 0 ? planes_at + planes : (tucker ? kFactorBytes : 0);
  if (st == UMEM_OK && need > 0 && (ws == nullptr || !aligned(ws, kAlign) || ws_bytes < need))
    st = UMEM_ERR_WORKSPACE;
  if (st != UMEM_OK) return st;
  float* factors = tucker ? static_cast<float*>(ws) : nullptr;
  hipError_t e = tucker ? launch_rank1(*desc, core, factors, stream) : hipSuccess;
  if (e == hipSuccess)
    e = launch_axis_scores(*desc, T, q_row, q_col, k_row, k_col, factors, sel, nullptr, 0,
                           planes > 0 ? static_cast<char*>(ws) + planes_at : nullptr, stream);
  return hip_status(e);
}

UMEM_API umem_status umem_select(const umem_desc* desc, int32_t T, const float* sel,
                                 const float* q_row, const float* q_col, const float* k_row,
                                 const float* k_col, const float* core, int32_t* idx, float* w,
                                 int32_t* axis_idx, const void* values, float* pooled,
                                 hipStream_t stream) {
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (st == UMEM_OK && desc->grid == UMEM_GRID_TUCKER)
    st = check_scoring_ptrs(desc, q_row, q_col, k_row, k_col, core);
  if (st == UMEM_OK && (!sel || !idx || !w || !aligned(sel, 16) || !aligned(idx, 4) || !aligned(w, 4) ||
                        !aligned(axis_idx, 4)))
    st = UMEM_ERR_INVALID_ARG;
  if (st == UMEM_OK && (values == nullptr) != (pooled == nullptr)) st = UMEM_ERR_INVALID_ARG;
  if (st == UMEM_OK && pooled != nullptr) {
    if (!aligned(values, 16) || !aligned(pooled, 16)) st = UMEM_ERR_INVALID_ARG;
    else if (!select_pools(*desc)) st = UMEM_ERR_UNSUPPORTED;
  }
  if (st != UMEM_OK) return st;
  return hip_status(launch_select(*desc, T, sel, q_row, q_col, k_row, k_col, core, idx, w,
                                  axis_idx, values, pooled, stream));
}

UMEM_API umem_status umem_score_topk(const umem_desc* desc, int32_t T, const float* q_row,
                                     const float* q_col, const float* k_row, const float* k_col,
                                     const float* core, int32_t* idx, float* w, int32_t* axis_idx,
                                     void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (st == UMEM_OK) st = check_scoring_ptrs(desc, q_row, q_col, k_row, k_col, core);
  if (st == UMEM_OK && (!idx || !w || !aligned(idx, 4) || !aligned(w, 4) || !aligned(axis_idx, 4)))
    st = UMEM_ERR_INVALID_ARG;
  if (st == UMEM_OK) st = check_ws(desc, T, ws, ws_bytes);
  if (st != UMEM_OK) return st;
  const Layout L = layout(desc, T);
  float* sel = reinterpret_cast<float*>(static_cast<char*>(ws) + L.sel);
  float* factors = reinterpret_cast<float*>(static_cast<char*>(ws) + L.factors);
  const bool tucker = desc->grid == UMEM_GRID_TUCKER;
  hipError_t e = tucker ? launch_rank1(*desc, core, factors, stream) : hipSuccess;
  if (e == hipSuccess)
    e = launch_axis_scores(*desc, T, q_row, q_col, k_row, k_col, tucker ? factors : nullptr, sel,
                           nullptr, 0, static_cast<char*>(ws) + L.proj, stream);
  if (e == hipSuccess)
    e = launch_select(*desc, T, sel, q_row, q_col, k_row, k_col, core, idx, w, axis_idx, nullptr,
                      nullptr, stream);
  return hip_status(e);
}

UMEM_API umem_status umem_gather_sum(int64_t n_values, int32_t dv, int32_t vdtype,
                                     const void* values, int32_t T, int32_t bag,
                                     const int32_t* idx, const float* w, const int32_t* perm,
                                     int32_t expand, int32_t cores, float* out,
                                     hipStream_t stream) {
  umem_status st = check_gather(n_values, dv, vdtype, values, T, bag, idx, w, expand, cores, out);
  if (st != UMEM_OK || T == 0) return st;
  if (st == UMEM_OK && perm != nullptr && !aligned(perm, 4)) st = UMEM_ERR_INVALID_ARG;
  if (st != UMEM_OK) return st;
  return hip_status(launch_gather(n_values, dv, vdtype, values, T, bag, idx, w, perm, expand,
                                  cores > 1 ? cores : 1, out, stream));
}

UMEM_API umem_status umem_project_workspace_size(int32_t T, int32_t expand, int32_t dv,
                                                 int32_t dv_virt, int32_t d_out, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  // the output linear alone has dv_virt == 0; with dv_virt > 0 the projector is given
  umem_status st = check_project_shape(expand, dv, dv_virt, d_out, dv_virt > 0, d_out > 0);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  *bytes = most_upto(T, [=](int32_t t) { return project_workspace_bytes(t, expand, dv, dv_virt, d_out); });
  return UMEM_OK;
}

UMEM_API umem_status umem_project(int32_t T, int32_t expand, int32_t dv, int32_t dv_virt,
                                  int32_t d_out, const float* pooled, const uint16_t* w_proj,
                                  const uint16_t* w_out, float* out, void* ws, size_t ws_bytes,
                                  hipStream_t stream) {
  umem_status st = check_project(T, expand, dv, dv_virt, d_out, pooled, w_proj, w_out, out, ws,
                                 ws_bytes);
  if (st != UMEM_OK || T == 0) return st;
  return hip_status(run_project(T, expand, dv, dv_virt, d_out, pooled, w_proj, w_out, out, ws, stream));
}

}  // extern "C"

namespace {

umem_status check_query_desc(const umem_query_desc* qd) {
  if (qd == nullptr) return UMEM_ERR_INVALID_ARG;
  if (qd->d_model < 1 || qd->conv_k < 1 || qd->heads < 1 || qd->dk < 1) return UMEM_ERR_INVALID_ARG;
  if ((qd->shared != 0 && qd->shared != 1) || !(qd->eps >= 0.0f) || qd->eps == INFINITY)
    return UMEM_ERR_INVALID_ARG;
  const int64_t nq = static_cast<int64_t>(qd->shared ? 1 : 2) * qd->heads * qd->dk;
  if (qd->d_model % 8 != 0 || qd->conv_k > 8 || qd->dk > 1024 || nq % 8 != 0 || nq > (1 << 24) ||
      !gemm_weight_supported(nq, qd->d_model))
    return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

umem_status check_query_ptrs(const umem_query_desc* qd, const float* x, const float* x_hist, const float* conv_w,
                             const uint16_t* w_q, const float* gamma, const float* beta, const float* q_row,
                             const float* q_col) {
  if (!x || !conv_w || !w_q || !gamma || !beta || !q_row) return UMEM_ERR_INVALID_ARG;
  if ((q_col == nullptr) != (qd->shared == 1)) return UMEM_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(x_hist, 16) || !aligned(conv_w, 16) || !aligned(w_q, 16))
    return UMEM_ERR_INVALID_ARG;
  if (!aligned(gamma, 4) || !aligned(beta, 4) || !aligned(q_row, 4) || !aligned(q_col, 4))
    return UMEM_ERR_INVALID_ARG;
  return UMEM_OK;
}

size_t query_workspace_most(const umem_query_desc& qd, int64_t T) {
  return most_upto(T, [&](int32_t t) { return query_workspace_bytes(qd, t); });
}

umem_status check_query_tokens(int32_t B, int32_t L) {
  if (B < 0 || L < 0) return UMEM_ERR_INVALID_ARG;
  if (static_cast<int64_t>(B) * L > kMaxTokens) return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_query_workspace_size(const umem_query_desc* qd, int32_t B, int32_t L,
                                               size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_query_desc(qd);
  if (st == UMEM_OK) st = check_query_tokens(B, L);
  if (st != UMEM_OK) return st;
  *bytes = query_workspace_most(*qd, static_cast<int64_t>(B) * L);
  return UMEM_OK;
}

UMEM_API umem_status umem_query(const umem_query_desc* qd, int32_t B, int32_t L, const float* x,
                                const float* x_hist, const float* conv_w, const uint16_t* w_q,
                                const float* gamma, const float* beta, float* q_row, float* q_col,
                                void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_query_desc(qd);
  if (st == UMEM_OK) st = check_query_tokens(B, L);
  if (st != UMEM_OK) return st;
  if (static_cast<int64_t>(B) * L == 0) return UMEM_OK;
  st = check_query_ptrs(qd, x, x_hist, conv_w, w_q, gamma, beta, q_row, q_col);
  if (st != UMEM_OK) return st;
  const size_t need = query_workspace_bytes(*qd, static_cast<int64_t>(B) * L);
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  return hip_status(launch_query(*qd, B, L, x, x_hist, conv_w, w_q, gamma, beta, q_row, q_col, ws,
                                 nullptr, stream));
}

UMEM_API umem_status umem_key_norm(int32_t heads, int32_t n, int32_t dk, const float* keys,
                                   const float* gamma, const float* beta, float eps, float* out,
                                   hipStream_t stream) {
  if (heads < 1 || n < 1 || dk < 1 || !(eps >= 0.0f) || eps == INFINITY) return UMEM_ERR_INVALID_ARG;
  if (!keys || !gamma || !beta || !out) return UMEM_ERR_INVALID_ARG;
  if (!aligned(keys, 4) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(out, 4))
    return UMEM_ERR_INVALID_ARG;
  if (dk > 1024 || static_cast<int64_t>(heads) * n > (INT64_C(1) << 31)) return UMEM_ERR_UNSUPPORTED;
  return hip_status(launch_key_norm(heads, n, dk, keys, gamma, beta, eps, out, stream));
}

constexpr int64_t kMaxBackwardEntries = INT64_C(1) << 22;   // pairs the backward sorts at once

UMEM_API umem_status umem_gather_backward_workspace_size(int32_t T, int32_t bag, int32_t dv,
                                                         size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  if (T < 0 || bag < 1 || dv < 1) return UMEM_ERR_INVALID_ARG;
  if (static_cast<int64_t>(T) * bag > kMaxBackwardEntries) return UMEM_ERR_UNSUPPORTED;
  *bytes = gather_backward_workspace_bytes(T, bag, dv);
  return UMEM_OK;
}

UMEM_API umem_status umem_gather_backward(int64_t n_values, int32_t dv, int32_t vdtype,
                                          const void* values, int32_t T, int32_t bag,
                                          const int32_t* idx, const float* w, const int32_t* perm,
                                          int32_t expand, int32_t cores, const float* d_pooled,
                                          float* d_values, float* dw, void* ws, size_t ws_bytes,
                                          hipStream_t stream) {
  umem_status st = check_gather(n_values, dv, vdtype, values, T, bag, idx, w, expand, cores, d_values);
  if (st != UMEM_OK || T == 0) return st;
  if (!d_pooled || !dw || !aligned(d_pooled, 16) || !aligned(dw, 4)) return UMEM_ERR_INVALID_ARG;
  if ((expand > 1) != (perm != nullptr) || !aligned(perm, 4)) return UMEM_ERR_INVALID_ARG;
  if (static_cast<int64_t>(T) * bag > kMaxBackwardEntries) return UMEM_ERR_UNSUPPORTED;
  const size_t need = gather_backward_workspace_bytes(T, bag, dv);
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  return hip_status(launch_gather_backward(n_values, dv, vdtype, values, T, bag, idx, w, perm,
                                           expand, cores, d_pooled, d_values, dw, nullptr, nullptr,
                                           ws, stream));
}

UMEM_API umem_status umem_gather_backward_rows(int64_t n_values, int32_t dv, int32_t vdtype,
                                               const void* values, int32_t T, int32_t bag,
                                               const int32_t* idx, const float* w,
                                               const int32_t* perm, int32_t expand, int32_t cores,
                                               const float* d_pooled, int32_t* rows, float* d_rows,
                                               int32_t* n_rows, float* dw, void* ws,
                                               size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_gather(n_values, dv, vdtype, values, T, bag, idx, w, expand, cores, d_rows);
  if (st != UMEM_OK || T == 0) return st;
  if (!rows || !n_rows || !aligned(rows, 4) || !aligned(n_rows, 4)) return UMEM_ERR_INVALID_ARG;
  if (!d_pooled || !dw || !aligned(d_pooled, 16) || !aligned(dw, 4)) return UMEM_ERR_INVALID_ARG;
  if ((expand > 1) != (perm != nullptr) || !aligned(perm, 4)) return UMEM_ERR_INVALID_ARG;
  if (static_cast<int64_t>(T) * bag > kMaxBackwardEntries) return UMEM_ERR_UNSUPPORTED;
  const size_t need = gather_backward_workspace_bytes(T, bag, dv);
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  return hip_status(launch_gather_backward(n_values, dv, vdtype, values, T, bag, idx, w, perm,
                                           expand, cores, d_pooled, d_rows, dw, rows, n_rows, ws,
                                           stream));
}

UMEM_API umem_status umem_score_backward_workspace_size(const umem_desc* desc, int32_t T,
                                                        size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  if (static_cast<int64_t>(T) * desc->heads * 2 * desc->topm > kMaxBackwardEntries)
    return UMEM_ERR_UNSUPPORTED;
  *bytes = score_backward_workspace_bytes(*desc, T);
  return UMEM_OK;
}

UMEM_API umem_status umem_score_backward(const umem_desc* desc, int32_t T, const float* q_row,
                                         const float* q_col, const float* k_row,
                                         const float* k_col, const float* core,
                                         const int32_t* idx, const float* w, const float* dw,
                                         float* dq_row, float* dq_col, float* dk_row,
                                         float* dk_col, float* dcore, void* ws, size_t ws_bytes,
                                         hipStream_t stream) {
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  st = check_scoring_ptrs(desc, q_row, q_col, k_row, k_col, core);
  if (st != UMEM_OK) return st;
  const bool softmax = desc->weight == UMEM_W_SOFTMAX;
  if (!idx || !dw || (softmax && !w)) return UMEM_ERR_INVALID_ARG;
  if (!aligned(idx, 4) || !aligned(dw, 4) || !aligned(w, 4)) return UMEM_ERR_INVALID_ARG;
  if (!dq_row || !dq_col || !dk_row || !dk_col) return UMEM_ERR_INVALID_ARG;
  if (!aligned(dq_row, 4) || !aligned(dq_col, 4) || !aligned(dk_row, 16) || !aligned(dk_col, 16))
    return UMEM_ERR_INVALID_ARG;
  if ((desc->grid == UMEM_GRID_TUCKER) != (dcore != nullptr) || !aligned(dcore, 4))
    return UMEM_ERR_INVALID_ARG;
  if (static_cast<int64_t>(T) * desc->heads * 2 * desc->topm > kMaxBackwardEntries)
    return UMEM_ERR_UNSUPPORTED;
  const size_t need = score_backward_workspace_bytes(*desc, T);
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  return hip_status(launch_score_backward(*desc, T, q_row, q_col, k_row, k_col, core, idx, w, dw,
                                          dq_row, dq_col, dk_row, dk_col, dcore, ws, stream));
}

}  // extern "C"

namespace {

bool finite(float x) { return x - x == 0.0f; }

size_t esize(int32_t dtype) { return dtype == UMEM_BF16 ? 2 : 4; }

bool known_type(int64_t dtype) { return dtype == UMEM_F32 || dtype == UMEM_BF16; }

// An array of a call, for the checks that outputs lie apart from what the kernels read meanwhile.
struct Span {
  const void* p;
  size_t bytes;
};

bool apart(const Span& a, const Span& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return true;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x + a.bytes <= y || y + b.bytes <= x;
}

// Whether `out` is apart from the n arrays in[], or is in[same] itself.
bool out_fits(const Span& out, const Span* in, int n, int same = -1) {
  for (int i = 0; i < n; ++i)
    if (!apart(out, in[i]) && !(i == same && out.p == in[i].p && out.bytes == in[i].bytes)) return false;
  return true;
}

umem_status check_block_desc(const umem_block_desc* bd) {
  if (bd == nullptr || bd->d < 1) return UMEM_ERR_INVALID_ARG;
  if (bd->norm_in != UMEM_NORM_LAYER && bd->norm_in != UMEM_NORM_RMS) return UMEM_ERR_INVALID_ARG;
  if (bd->norm_out < UMEM_NORM_LAYER || bd->norm_out > UMEM_NORM_NONE) return UMEM_ERR_INVALID_ARG;
  if (bd->gate < UMEM_GATE_NONE || bd->gate > UMEM_GATE_FULL) return UMEM_ERR_INVALID_ARG;
  if (bd->gate_act != UMEM_ACT_LINEAR && bd->gate_act != UMEM_ACT_SIGMOID) return UMEM_ERR_INVALID_ARG;
  if (!known_type(bd->htype) || !known_type(bd->ytype)) return UMEM_ERR_INVALID_ARG;
  if (!finite(bd->eps) || bd->eps < 0.0f || !finite(bd->res_scale) || !finite(bd->out_scale))
    return UMEM_ERR_INVALID_ARG;
  if (bd->d > kMaxBlockWidth) return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

// The arrays of a block call: [T, d] of the stream's or the block's type, fp32 [d], the gate.
struct BlockSpans {
  size_t h, y, row, gate;
  int32_t gate_type;
  BlockSpans(const umem_block_desc& bd, int32_t T) {
    const size_t n = static_cast<size_t>(T) * bd.d;
    h = n * esize(bd.htype);
    y = n * esize(bd.ytype);
    row = static_cast<size_t>(bd.d) * 4;
    gate_type = bd.gate == UMEM_GATE_FULL ? bd.ytype : UMEM_F32;
    gate = bd.gate == UMEM_GATE_FULL ? y : bd.gate == UMEM_GATE_TOKEN ? static_cast<size_t>(T) * 4 : row;
  }
};

umem_status check_block_ws(const umem_block_desc& bd, int32_t T, const void* ws, size_t ws_bytes) {
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < block_backward_workspace_bytes(bd, T)) return UMEM_ERR_WORKSPACE;
  return UMEM_OK;
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_block_in(const umem_block_desc* bd, int32_t T, const void* h, const float* gamma,
                                   const float* beta, void* n, hipStream_t stream) {
  umem_status st = check_block_desc(bd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!h || !gamma || !n) return UMEM_ERR_INVALID_ARG;
  const BlockSpans z(*bd, T);
  if (!aligned(h, esize(bd->htype)) || !aligned(n, esize(bd->ytype)) || !aligned(gamma, 4) || !aligned(beta, 4))
    return UMEM_ERR_INVALID_ARG;
  const Span in[] = {{h, z.h}, {gamma, z.row}, {beta, z.row}};
  if (!out_fits({n, z.y}, in, 3, 0)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_block_in(*bd, T, h, gamma, beta, n, stream));
}

UMEM_API umem_status umem_block_out(const umem_block_desc* bd, int32_t T, const void* h, const void* y,
                                    const void* gate, const float* gamma, const float* beta, void* h_out,
                                    const float* gamma_next, const float* beta_next, void* n_next,
                                    hipStream_t stream) {
  umem_status st = check_block_desc(bd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!h || !y || !h_out) return UMEM_ERR_INVALID_ARG;
  if ((gate != nullptr) != (bd->gate != UMEM_GATE_NONE)) return UMEM_ERR_INVALID_ARG;
  if ((gamma != nullptr) != (bd->norm_out != UMEM_NORM_NONE) || (beta && !gamma)) return UMEM_ERR_INVALID_ARG;
  if ((gamma_next != nullptr) != (n_next != nullptr) || (beta_next && !n_next)) return UMEM_ERR_INVALID_ARG;
  const BlockSpans z(*bd, T);
  if (!aligned(h, esize(bd->htype)) || !aligned(h_out, esize(bd->htype)) || !aligned(y, esize(bd->ytype)) ||
      !aligned(n_next, esize(bd->ytype)) || !aligned(gate, esize(z.gate_type)) || !aligned(gamma, 4) ||
      !aligned(beta, 4) || !aligned(gamma_next, 4) || !aligned(beta_next, 4))
    return UMEM_ERR_INVALID_ARG;
  const Span in[] = {{h, z.h},       {y, z.y},           {gate, z.gate},      {gamma, z.row},
                     {beta, z.row}, {gamma_next, z.row}, {beta_next, z.row}};
  if (!out_fits({h_out, z.h}, in, 7, 0) || !out_fits({n_next, z.y}, in, 7, 1) || !apart({h_out, z.h}, {n_next, z.y}))
    return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_block_out(*bd, T, h, y, gate, gamma, beta, h_out, gamma_next, beta_next, n_next, stream));
}

UMEM_API umem_status umem_block_backward_workspace_size(const umem_block_desc* bd, int32_t T, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_block_desc(bd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  *bytes = block_backward_workspace_bytes(*bd, T);
  return UMEM_OK;
}

UMEM_API umem_status umem_block_in_backward(const umem_block_desc* bd, int32_t T, const void* h, const float* gamma,
                                            const void* dn, const void* dres, void* dh, float* dgamma,
                                            float* dbeta, int32_t accumulate, void* ws, size_t ws_bytes,
                                            hipStream_t stream) {
  umem_status st = check_block_desc(bd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  if (accumulate != 0 && accumulate != 1) return UMEM_ERR_INVALID_ARG;
  if (T == 0) return UMEM_OK;
  if (!h || !gamma || !dn || !dh || !dgamma) return UMEM_ERR_INVALID_ARG;
  const size_t hs = esize(bd->htype);
  if (!aligned(h, hs) || !aligned(dres, hs) || !aligned(dh, hs) || !aligned(dn, esize(bd->ytype)) ||
      !aligned(gamma, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return UMEM_ERR_INVALID_ARG;
  st = check_block_ws(*bd, T, ws, ws_bytes);
  if (st != UMEM_OK) return st;
  const BlockSpans z(*bd, T);
  const Span in[] = {{h, z.h}, {dres, z.h}, {dn, z.y}, {gamma, z.row},
                     {ws, block_backward_workspace_bytes(*bd, T)}};
  const Span dx{dh, z.h}, dg{dgamma, z.row}, db{dbeta, z.row};
  if (!out_fits(in[4], in, 4)) return UMEM_ERR_INVALID_ARG;          // the scratch is written while they are read
  if ((!out_fits(dx, in, 5, 0) && !out_fits(dx, in, 5, 1)) || !out_fits(dg, in, 5) || !out_fits(db, in, 5) ||
      !apart(dx, dg) || !apart(dx, db) || !apart(dg, db))
    return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_block_in_backward(*bd, T, h, gamma, dn, dres, dh, dgamma, dbeta, accumulate != 0, ws,
                                             stream));
}

UMEM_API umem_status umem_block_out_backward(const umem_block_desc* bd, int32_t T, const void* y, const void* gate,
                                             const float* gamma, const float* beta, const void* dh_out, void* dh,
                                             void* dy, void* dgate, float* dgamma, float* dbeta,
                                             int32_t accumulate, void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_block_desc(bd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  if (accumulate != 0 && accumulate != 1) return UMEM_ERR_INVALID_ARG;
  if (T == 0) return UMEM_OK;
  if (!y || !dh_out || !dy) return UMEM_ERR_INVALID_ARG;
  const bool gated = bd->gate != UMEM_GATE_NONE, normed = bd->norm_out != UMEM_NORM_NONE;
  if ((gate != nullptr) != gated || (dgate != nullptr) != gated) return UMEM_ERR_INVALID_ARG;
  if ((gamma != nullptr) != normed || (dgamma != nullptr) != normed) return UMEM_ERR_INVALID_ARG;
  if ((beta && !gamma) || (beta != nullptr) != (dbeta != nullptr)) return UMEM_ERR_INVALID_ARG;
  const BlockSpans z(*bd, T);
  const size_t hs = esize(bd->htype), ys = esize(bd->ytype), gs = esize(z.gate_type);
  if (!aligned(y, ys) || !aligned(dy, ys) || !aligned(dh_out, hs) || !aligned(dh, hs) || !aligned(gate, gs) ||
      !aligned(dgate, gs) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return UMEM_ERR_INVALID_ARG;
  st = check_block_ws(*bd, T, ws, ws_bytes);
  if (st != UMEM_OK) return st;
  const Span in[] = {{y, z.y},       {dh_out, z.h}, {gate, z.gate},
                     {gamma, z.row}, {beta, z.row}, {ws, block_backward_workspace_bytes(*bd, T)}};
  const Span out[] = {{dy, z.y}, {dh, z.h}, {dgate, z.gate}, {dgamma, z.row}, {dbeta, z.row}};
  const int same[] = {0, 1, bd->gate == UMEM_GATE_FULL ? 2 : -1, -1, -1};
  if (!out_fits(in[5], in, 5)) return UMEM_ERR_INVALID_ARG;
  for (int i = 0; i < 5; ++i)
    if (!out_fits(out[i], in, 6, same[i]) || !out_fits(out[i], out, i)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_block_out_backward(*bd, T, y, gate, gamma, beta, dh_out, dh, dy, dgate, dgamma, dbeta,
                                              accumulate != 0, ws, stream));
}

}  // extern "C"

namespace {

// for_clip: the outs are written, so they are checked as well.
umem_status check_grads(int32_t n, const umem_grad* grads, bool for_clip) {
  if (n < 0 || (n > 0 && grads == nullptr)) return UMEM_ERR_INVALID_ARG;
  if (n > kMaxGrads) return UMEM_ERR_UNSUPPORTED;
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    const umem_grad& g = grads[i];
    if (g.rows < 0 || g.row_len < 0 || !known_type(g.dtype)) return UMEM_ERR_INVALID_ARG;
    if (g.rows == 0 || g.row_len == 0) continue;
    constexpr int64_t kMost = INT64_C(1) << 40;
    if (g.rows > kMost / g.row_len) return UMEM_ERR_UNSUPPORTED;
    total += g.rows * g.row_len;
    if (total > kMost) return UMEM_ERR_UNSUPPORTED;
    const size_t es = esize(static_cast<int32_t>(g.dtype));
    if (g.grad == nullptr || !aligned(g.grad, es) || !aligned(g.n_rows, 4)) return UMEM_ERR_INVALID_ARG;
    if (for_clip && (g.out == nullptr || !aligned(g.out, es))) return UMEM_ERR_INVALID_ARG;
  }
  return UMEM_OK;
}

// Whether what the norm writes (itself, the sum of squares, the scratch) overlaps a gradient, a row count or each other.
bool norm_clashes(int32_t n, const umem_grad* grads, const Span& norm, const Span& sumsq, const Span& ws) {
  const Span out[] = {norm, sumsq, ws};
  if (!apart(norm, sumsq) || !apart(norm, ws) || !apart(sumsq, ws)) return true;
  for (int i = 0; i < n; ++i) {
    const umem_grad& g = grads[i];
    const Span in{g.grad, static_cast<size_t>(g.rows) * g.row_len * esize(static_cast<int32_t>(g.dtype))};
    if (in.bytes == 0) continue;
    const Span rows{g.n_rows, sizeof(int32_t)};
    for (const Span& o : out)
      if (!apart(o, in) || !apart(o, rows)) return true;
  }
  return false;
}

// Whether an out overlaps another gradient or out, its own gradient other than being it, or what the kernels
// read beside them: the norm and the row counts.
bool grads_clash(int32_t n, const umem_grad* grads, const float* norm) {
  struct Range {
    uintptr_t from, to;
  };
  static_assert((3 * kMaxGrads + 1) * sizeof(Range) <= 128 << 10, "the ranges live on the caller's stack");
  Range out[kMaxGrads], in[2 * kMaxGrads + 1];
  int outs = 0, ins = 0;
  for (int i = 0; i < n; ++i) {
    const umem_grad& g = grads[i];
    const uintptr_t bytes = static_cast<uintptr_t>(g.rows) * g.row_len * esize(static_cast<int32_t>(g.dtype));
    if (bytes == 0) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(g.grad), b = reinterpret_cast<uintptr_t>(g.out);
    out[outs++] = {b, b + bytes};
    if (a != b) in[ins++] = {a, a + bytes};
    const uintptr_t rows = reinterpret_cast<uintptr_t>(g.n_rows);
    if (rows != 0 && (ins == 0 || in[ins - 1].from != rows)) in[ins++] = {rows, rows + sizeof(int32_t)};
  }
  in[ins++] = {reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm) + sizeof(float)};
  const auto before = [](const Range& a, const Range& b) { return a.from < b.from; };
  if (!std::is_sorted(out, out + outs, before)) std::sort(out, out + outs, before);
  if (!std::is_sorted(in, in + ins, before)) std::sort(in, in + ins, before);
  for (int i = 1; i < outs; ++i)
    if (out[i].from < out[i - 1].to) return true;
  // the outs are apart: a gradient meets the last that starts at or before it, or the next
  for (int i = 0, j = 0; i < ins; ++i) {
    while (j < outs && out[j].from <= in[i].from) ++j;
    if ((j > 0 && out[j - 1].to > in[i].from) || (j < outs && out[j].from < in[i].to)) return true;
  }
  return false;
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_grad_workspace_size(int32_t n, const umem_grad* grads, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  const umem_status st = check_grads(n, grads, false);
  if (st != UMEM_OK) return st;
  *bytes = grad_workspace_bytes(n, grads);
  return UMEM_OK;
}

UMEM_API umem_status umem_grad_norm(int32_t n, const umem_grad* grads, float* norm, double* sumsq, void* ws,
                                    size_t ws_bytes, hipStream_t stream) {
  const umem_status st = check_grads(n, grads, false);
  if (st != UMEM_OK) return st;
  if (norm == nullptr || !aligned(norm, 4) || !aligned(sumsq, 8)) return UMEM_ERR_INVALID_ARG;
  const size_t need = grad_workspace_bytes(n, grads);
  if (norm_clashes(n, grads, {norm, sizeof(float)}, {sumsq, sizeof(double)}, {ws, need})) return UMEM_ERR_INVALID_ARG;
  if (need > 0 && (ws == nullptr || !aligned(ws, 16) || ws_bytes < need)) return UMEM_ERR_WORKSPACE;
  return hip_status(launch_grad_norm(n, grads, norm, sumsq, ws, stream));
}

UMEM_API umem_status umem_grad_clip(int32_t n, const umem_grad* grads, float max_norm, const float* norm,
                                    hipStream_t stream) {
  const umem_status st = check_grads(n, grads, true);
  if (st != UMEM_OK) return st;
  if (!(max_norm >= 0.0f) || norm == nullptr || !aligned(norm, 4) || grads_clash(n, grads, norm)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_grad_clip(n, grads, max_norm, norm, stream));
}

}  // extern "C"

namespace {

umem_status check_adapter_desc(const umem_adapter_desc* ad) {
  if (ad == nullptr || ad->n < 1 || ad->rank < 1 || ad->d_in < 1 || ad->d_out < 1) return UMEM_ERR_INVALID_ARG;
  if (!known_type(ad->xtype) || !known_type(ad->otype)) return UMEM_ERR_INVALID_ARG;
  if (ad->rank % 8 != 0 || ad->d_in % 8 != 0 || ad->d_out % 8 != 0 || ad->rank > kMaxAdapterRank ||
      ad->d_in > kMaxAdapterWidth || ad->d_out > kMaxAdapterWidth)
    return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_adapter_workspace_size(const umem_adapter_desc* ad, int32_t T, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_adapter_desc(ad);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  *bytes = adapter_workspace_bytes(*ad, T);
  return UMEM_OK;
}

UMEM_API umem_status umem_adapter_add(const umem_adapter_desc* ad, int32_t T, const void* x, const int32_t* ids,
                                      const uint16_t* a, const uint16_t* b, const float* scale, const void* base,
                                      void* out, void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_adapter_desc(ad);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!x || !ids || !a || !b || !out) return UMEM_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(a, 16) || !aligned(b, 16) || !aligned(base, 16) || !aligned(out, 16) ||
      !aligned(ids, 4) || !aligned(scale, 4))
    return UMEM_ERR_INVALID_ARG;
  const size_t need = adapter_workspace_bytes(*ad, T);
  if (need > 0 && (ws == nullptr || !aligned(ws, kAlign) || ws_bytes < need)) return UMEM_ERR_WORKSPACE;
  const size_t t = T, n = ad->n, r = ad->rank;
  const Span y{out, t * ad->d_out * esize(ad->otype)};
  const Span in[] = {{base, y.bytes},          {x, t * ad->d_in * esize(ad->xtype)},
                     {ids, t * 4},             {a, n * r * ad->d_in * 2},
                     {b, n * ad->d_out * r * 2}, {scale, n * 4},
                     {ws, need}};
  if (!out_fits(y, in, 7, 0) || !out_fits(in[6], in, 6)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_adapter_add(*ad, T, x, ids, a, b, scale, base, out, ws, stream));
}

}  // extern "C"

namespace {

umem_status check_query_adapters(const umem_query_desc* qd, const umem_adapter_desc* ad, int32_t B, int32_t L) {
  umem_status st = check_query_desc(qd);
  if (st == UMEM_OK) st = check_adapter_desc(ad);
  if (st == UMEM_OK) st = check_query_tokens(B, L);
  if (st != UMEM_OK) return st;
  const int64_t nq = static_cast<int64_t>(qd->shared ? 1 : 2) * qd->heads * qd->dk;
  if (ad->d_in != qd->d_model || ad->d_out != nq || ad->xtype != UMEM_BF16 || ad->otype != UMEM_F32)
    return UMEM_ERR_INVALID_ARG;
  return UMEM_OK;
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_query_adapted_workspace_size(const umem_query_desc* qd, const umem_adapter_desc* ad,
                                                       int32_t B, int32_t L, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  const umem_status st = check_query_adapters(qd, ad, B, L);
  if (st != UMEM_OK) return st;
  const int64_t T = static_cast<int64_t>(B) * L;
  *bytes = round_up(query_workspace_most(*qd, T)) + adapter_workspace_bytes(*ad, static_cast<int>(T));
  return UMEM_OK;
}

UMEM_API umem_status umem_query_adapted(const umem_query_desc* qd, const umem_adapter_desc* ad, int32_t B, int32_t L,
                                        const float* x, const float* x_hist, const float* conv_w,
                                        const uint16_t* w_q, const int32_t* ids, const uint16_t* a,
                                        const uint16_t* b, const float* scale, const float* gamma,
                                        const float* beta, float* q_row, float* q_col, void* ws, size_t ws_bytes,
                                        hipStream_t stream) {
  umem_status st = check_query_adapters(qd, ad, B, L);
  if (st != UMEM_OK) return st;
  const int64_t T = static_cast<int64_t>(B) * L;
  if (T == 0) return UMEM_OK;
  st = check_query_ptrs(qd, x, x_hist, conv_w, w_q, gamma, beta, q_row, q_col);
  if (st != UMEM_OK) return st;
  if (!ids || !a || !b || !aligned(ids, 4) || !aligned(a, 16) || !aligned(b, 16) || !aligned(scale, 4))
    return UMEM_ERR_INVALID_ARG;
  const size_t own = round_up(query_workspace_bytes(*qd, T));
  const size_t need = own + adapter_workspace_bytes(*ad, static_cast<int>(T));
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  const size_t t = T, d = qd->d_model, nq = ad->d_out, half = t * qd->heads * qd->dk * 4, na = ad->n, r = ad->rank;
  const Span in[] = {{x, t * d * 4},   {x_hist, static_cast<size_t>(B) * (qd->conv_k - 1) * d * 4},
                     {conv_w, qd->conv_k * d * 4}, {w_q, nq * d * 2}, {ids, t * 4},
                     {a, na * r * d * 2}, {b, na * nq * r * 2}, {scale, na * 4},
                     {gamma, nq * 4},  {beta, nq * 4}};
  const Span out[] = {{q_row, half}, {q_col, half}, {ws, need}};
  for (int i = 0; i < 3; ++i)
    if (!out_fits(out[i], in, 10) || !out_fits(out[i], out, i)) return UMEM_ERR_INVALID_ARG;
  const QueryAdapters adapters{*ad, ids, a, b, scale, static_cast<char*>(ws) + own};
  return hip_status(launch_query(*qd, B, L, x, x_hist, conv_w, w_q, gamma, beta, q_row, q_col, ws, &adapters, stream));
}

}  // extern "C"

namespace {

umem_status check_embed_desc(const umem_embed_desc* ed) {
  if (ed == nullptr || ed->vocab < 1 || ed->d < 1 || !known_type(ed->wtype) || !known_type(ed->otype) ||
      !finite(ed->scale))
    return UMEM_ERR_INVALID_ARG;
  return ed->d > kMaxModelWidth ? UMEM_ERR_UNSUPPORTED : UMEM_OK;
}

// The gradient calls' checks: in[] ids, dout; out[] what the call writes beside ws.
umem_status check_embed_backward(const umem_embed_desc* ed, int32_t T, const int32_t* ids, const void* dout,
                                 const Span* out, int outs, const void* ws, size_t ws_bytes) {
  if (!ids || !dout || !aligned(ids, 4) || !aligned(dout, esize(ed->otype))) return UMEM_ERR_INVALID_ARG;
  const size_t need = embed_backward_workspace_bytes(*ed, T), t = T;
  if (ws == nullptr || !aligned(ws, 16) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  const Span in[] = {{ids, t * 4}, {dout, t * ed->d * esize(ed->otype)}, {ws, need}};
  if (!out_fits(in[2], in, 2)) return UMEM_ERR_INVALID_ARG;
  for (int i = 0; i < outs; ++i)
    if (!out_fits(out[i], in, 3) || !out_fits(out[i], out, i)) return UMEM_ERR_INVALID_ARG;
  return UMEM_OK;
}

umem_status check_head_desc(const umem_head_desc* hd) {
  if (hd == nullptr || hd->vocab < 1 || hd->d < 1 || !known_type(hd->xtype) || !known_type(hd->gtype) ||
      !finite(hd->scale))
    return UMEM_ERR_INVALID_ARG;
  if (hd->d % 8 != 0 || hd->d > kMaxModelWidth || hd->vocab > kMaxHeadVocab) return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

umem_status check_orth_desc(const umem_orth_desc* od) {
  if (od == nullptr || od->n < 1 || od->rows < 1 || od->cols < 1 || od->steps < 1 || !known_type(od->gtype) ||
      !known_type(od->otype))
    return UMEM_ERR_INVALID_ARG;
  if (!finite(od->a) || !finite(od->b) || !finite(od->c) || !finite(od->eps) || od->eps < 0.0f || !finite(od->decay) ||
      !finite(od->scale))
    return UMEM_ERR_INVALID_ARG;
  if (od->rows > kMaxOrthSide || od->cols > kMaxOrthSide || od->n > kMaxOrthBatch || od->steps > kMaxOrthSteps ||
      static_cast<int64_t>(od->rows) * od->cols > kMaxOrthElements / od->n)
    return UMEM_ERR_UNSUPPORTED;
  return UMEM_OK;
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_embed(const umem_embed_desc* ed, int32_t T, const void* table, const int32_t* ids, void* out,
                                hipStream_t stream) {
  umem_status st = check_embed_desc(ed);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!table || !ids || !out) return UMEM_ERR_INVALID_ARG;
  if (!aligned(table, esize(ed->wtype)) || !aligned(ids, 4) || !aligned(out, esize(ed->otype)))
    return UMEM_ERR_INVALID_ARG;
  const size_t t = T, d = ed->d;
  const Span in[] = {{table, static_cast<size_t>(ed->vocab) * d * esize(ed->wtype)}, {ids, t * 4}};
  if (!out_fits({out, t * d * esize(ed->otype)}, in, 2)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_embed(*ed, T, table, ids, out, stream));
}

UMEM_API umem_status umem_embed_backward_workspace_size(const umem_embed_desc* ed, int32_t T, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_embed_desc(ed);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  *bytes = embed_backward_workspace_bytes(*ed, T);
  return UMEM_OK;
}

UMEM_API umem_status umem_embed_backward(const umem_embed_desc* ed, int32_t T, const int32_t* ids, const void* dout,
                                         float* dtable, void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_embed_desc(ed);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!dtable || !aligned(dtable, 4)) return UMEM_ERR_INVALID_ARG;
  const Span out[] = {{dtable, static_cast<size_t>(ed->vocab) * ed->d * 4}};
  st = check_embed_backward(ed, T, ids, dout, out, 1, ws, ws_bytes);
  if (st != UMEM_OK) return st;
  return hip_status(launch_embed_backward(*ed, T, ids, dout, dtable, nullptr, nullptr, ws, stream));
}

UMEM_API umem_status umem_embed_backward_rows(const umem_embed_desc* ed, int32_t T, const int32_t* ids,
                                              const void* dout, int32_t* rows, float* d_rows, int32_t* n_rows, void* ws,
                                              size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_embed_desc(ed);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!rows || !d_rows || !n_rows || !aligned(rows, 4) || !aligned(d_rows, 4) || !aligned(n_rows, 4))
    return UMEM_ERR_INVALID_ARG;
  const size_t t = T;
  const Span out[] = {{rows, t * 4}, {d_rows, t * ed->d * 4}, {n_rows, 4}};
  st = check_embed_backward(ed, T, ids, dout, out, 3, ws, ws_bytes);
  if (st != UMEM_OK) return st;
  return hip_status(launch_embed_backward(*ed, T, ids, dout, d_rows, rows, n_rows, ws, stream));
}

UMEM_API umem_status umem_head_loss_workspace_size(const umem_head_desc* hd, int32_t T, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_head_desc(hd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  *bytes = head_loss_workspace_bytes(*hd, T);
  return UMEM_OK;
}

UMEM_API umem_status umem_head_loss(const umem_head_desc* hd, int32_t T, const void* x, const uint16_t* w,
                                    const int32_t* targets, float* loss, float* lse, void* ws, size_t ws_bytes,
                                    hipStream_t stream) {
  umem_status st = check_head_desc(hd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (!x || !w || !targets || !loss || !lse) return UMEM_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(targets, 4) || !aligned(loss, 4) || !aligned(lse, 4))
    return UMEM_ERR_INVALID_ARG;
  const size_t need = head_loss_workspace_bytes(*hd, T), t = T, d = hd->d;
  if (ws == nullptr || !aligned(ws, kAlign) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  const Span in[] = {{x, t * d * esize(hd->xtype)}, {w, static_cast<size_t>(hd->vocab) * d * 2}, {targets, t * 4}};
  const Span out[] = {{loss, t * 4}, {lse, t * 4}, {ws, need}};
  for (int i = 0; i < 3; ++i)
    if (!out_fits(out[i], in, 3) || !out_fits(out[i], out, i)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_head_loss(*hd, T, x, w, targets, loss, lse, ws, stream));
}

UMEM_API umem_status umem_head_backward_workspace_size(const umem_head_desc* hd, int32_t T, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  umem_status st = check_head_desc(hd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  *bytes = head_backward_workspace_bytes(*hd, T);
  return UMEM_OK;
}

UMEM_API umem_status umem_head_backward(const umem_head_desc* hd, int32_t T, const void* x, const uint16_t* w,
                                        const int32_t* targets, const float* lse, const float* dloss, void* dx,
                                        void* dw, int32_t accumulate, void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_head_desc(hd);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK) return st;
  if (accumulate != 0 && (accumulate != 1 || hd->gtype != UMEM_F32)) return UMEM_ERR_INVALID_ARG;
  if (T == 0) return UMEM_OK;
  if (!x || !w || !targets || !lse || !dx || !dw) return UMEM_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(dx, 16) || !aligned(dw, 16) || !aligned(targets, 4) ||
      !aligned(lse, 4) || !aligned(dloss, 4))
    return UMEM_ERR_INVALID_ARG;
  const size_t need = head_backward_workspace_bytes(*hd, T), t = T, d = hd->d, v = hd->vocab;
  if (ws == nullptr || !aligned(ws, kAlign) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  const Span in[] = {{x, t * d * esize(hd->xtype)}, {w, v * d * 2}, {targets, t * 4}, {lse, t * 4}, {dloss, t * 4}};
  const Span out[] = {{dx, t * d * esize(hd->xtype)}, {dw, v * d * esize(hd->gtype)}, {ws, need}};
  for (int i = 0; i < 3; ++i)
    if (!out_fits(out[i], in, 5) || !out_fits(out[i], out, i)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_head_backward(*hd, T, x, w, targets, lse, dloss, dx, dw, accumulate != 0, ws, stream));
}

UMEM_API umem_status umem_orthogonalize_workspace_size(const umem_orth_desc* od, size_t* bytes) {
  if (bytes == nullptr) return UMEM_ERR_INVALID_ARG;
  *bytes = 0;
  const umem_status st = check_orth_desc(od);
  if (st != UMEM_OK) return st;
  *bytes = orth_workspace_bytes(*od);
  return UMEM_OK;
}

UMEM_API umem_status umem_orthogonalize(const umem_orth_desc* od, const void* g, void* out, void* ws, size_t ws_bytes,
                                        hipStream_t stream) {
  const umem_status st = check_orth_desc(od);
  if (st != UMEM_OK) return st;
  if (!g || !out || !aligned(g, esize(od->gtype)) || !aligned(out, esize(od->otype))) return UMEM_ERR_INVALID_ARG;
  const size_t need = orth_workspace_bytes(*od), e = static_cast<size_t>(od->n) * od->rows * od->cols;
  if (ws == nullptr || !aligned(ws, kAlign) || ws_bytes < need) return UMEM_ERR_WORKSPACE;
  const Span in[] = {{g, e * esize(od->gtype)}, {ws, need}};
  if (!apart(in[0], in[1]) || !out_fits({out, e * esize(od->otype)}, in, 2, 0)) return UMEM_ERR_INVALID_ARG;
  return hip_status(launch_orthogonalize(*od, g, out, ws, stream));
}

}  // extern "C"

namespace {

umem_status forward_into(const umem_desc* desc, int32_t T, const float* q_row, const float* q_col,
                         const float* k_row, const float* k_col, const float* core,
                         const void* values, const int32_t* perm, const uint16_t* w_proj,
                         const uint16_t* w_out, float* out, int32_t* idx_out, float* w_out_scores,
                         void* ws, size_t ws_bytes, hipStream_t stream) {
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  if (st == UMEM_OK) st = check_scoring_ptrs(desc, q_row, q_col, k_row, k_col, core);
  if (st == UMEM_OK) st = check_ws(desc, T, ws, ws_bytes);
  if (st != UMEM_OK) return st;
  const bool project = desc->dv_virt > 0 || desc->d_out > 0;
  if ((desc->expand > 1) != (perm != nullptr)) return UMEM_ERR_INVALID_ARG;
  if ((desc->dv_virt > 0) != (w_proj != nullptr) || (desc->d_out > 0) != (w_out != nullptr))
    return UMEM_ERR_INVALID_ARG;
  if (!aligned(idx_out, 4) || !aligned(w_out_scores, 4) || !aligned(perm, 4))
    return UMEM_ERR_INVALID_ARG;
  if (!aligned(w_proj, 16) || !aligned(w_out, 16)) return UMEM_ERR_UNSUPPORTED;
  const int bag = desc->heads * desc->topm;
  const Layout L = layout(desc, T);
  char* base = static_cast<char*>(ws);
  float* sel = reinterpret_cast<float*>(base + L.sel);
  int32_t* idx = idx_out ? idx_out : reinterpret_cast<int32_t*>(base + L.idx);
  float* w = w_out_scores ? w_out_scores : reinterpret_cast<float*>(base + L.w);
  // with a projection the pooled rows go to the workspace in bf16, as its GEMM takes them
  uint16_t* pooled = reinterpret_cast<uint16_t*>(base + L.pooled);
  st = check_gather(desc->n_values, desc->dv, desc->vdtype, values, T, bag, idx, w, desc->expand,
                    n_cores(*desc), out);
  if (st != UMEM_OK) return st;

  float* factors = reinterpret_cast<float*>(base + L.factors);
  const bool tucker = desc->grid == UMEM_GRID_TUCKER;
  hipError_t e = tucker ? launch_rank1(*desc, core, factors, stream) : hipSuccess;
  // For decode-sized batches without expansion or projection the selection pools the rows
  // itself (scoring clears out first); otherwise the gather kernel, with more rows in flight per
  // CU, pools them after it.
  const bool fused = !project && select_pools(*desc) && T <= kMaxPoolTokens;
  if (e == hipSuccess)
    e = launch_axis_scores(*desc, T, q_row, q_col, k_row, k_col, tucker ? factors : nullptr, sel,
                           fused ? out : nullptr, static_cast<size_t>(T) * desc->dv,
                           base + L.proj, stream);
  if (e == hipSuccess)
    e = launch_select(*desc, T, sel, q_row, q_col, k_row, k_col, core, idx, w, nullptr,
                      fused ? values : nullptr, fused ? out : nullptr, stream);
  if (e == hipSuccess && !fused && !project)
    e = launch_gather(desc->n_values, desc->dv, desc->vdtype, values, T, bag, idx, w, perm,
                      desc->expand, n_cores(*desc), out, stream);
  if (e == hipSuccess && project)
    e = launch_gather_bf16(desc->n_values, desc->dv, desc->vdtype, values, T, bag, idx, w, perm,
                           desc->expand, n_cores(*desc), pooled, stream);
  if (e == hipSuccess && project)
    e = launch_project(T, desc->expand, desc->dv, desc->dv_virt, desc->d_out, pooled, w_proj,
                       w_out, out, base + L.proj, stream);
  return hip_status(e);
}

// The scratch of umem_forward_noalloc: one array in each GPU's memory, loaded with the library's
// code and held until the process ends.  Host code must not pass its name to a kernel (on the
// host it is only a stand-in for the device symbol); the device address of each GPU's copy is
// looked up once per device and kept in static_scratch_ptr.
static __device__ __align__(256) unsigned char scratch[UMEM_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::once_flag scratch_once[kMaxDevices];
void* scratch_ptr[kMaxDevices];
hipError_t scratch_err[kMaxDevices];

// The address of the current device's copy of `scratch` (its first call on a device looks it
// up, with that device current).
hipError_t static_scratch_ptr(void** ptr) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::call_once(scratch_once[dev], [dev] {
    void* p = nullptr;
    const hipError_t r = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    scratch_err[dev] = r;
    scratch_ptr[dev] = r == hipSuccess ? p : nullptr;
  });
  *ptr = scratch_ptr[dev];
  return scratch_err[dev];
}

}  // namespace

extern "C" {

UMEM_API umem_status umem_forward(const umem_desc* desc, int32_t T, const float* q_row,
                                  const float* q_col, const float* k_row, const float* k_col,
                                  const float* core, const void* values, const int32_t* perm,
                                  const uint16_t* w_proj, const uint16_t* w_out, float* out,
                                  int32_t* idx_out, float* w_out_scores, void* ws,
                                  size_t ws_bytes, hipStream_t stream) {
  return forward_into(desc, T, q_row, q_col, k_row, k_col, core, values, perm, w_proj, w_out, out,
                      idx_out, w_out_scores, ws, ws_bytes, stream);
}

UMEM_API umem_status umem_forward_noalloc(const umem_desc* desc, int32_t T, const float* q_row,
                                          const float* q_col, const float* k_row,
                                          const float* k_col, const float* core,
                                          const void* values, const int32_t* perm,
                                          const uint16_t* w_proj, const uint16_t* w_out,
                                          float* out, int32_t* idx_out, float* w_out_scores,
                                          hipStream_t stream) {
  umem_status st = check_desc(desc);
  if (st == UMEM_OK) st = check_tokens(T);
  if (st != UMEM_OK || T == 0) return st;
  // no kernel of the forward needs its scratch cleared beforehand: every part is written before
  // it is read, so the contents a previous call left behind do not matter
  if (layout(desc, T).total > UMEM_STATIC_SCRATCH_BYTES) return UMEM_ERR_SCRATCH_LIMIT;
  st = check_scoring_ptrs(desc, q_row, q_col, k_row, k_col, core);
  if (st != UMEM_OK) return st;
  void* ws = nullptr;
  if (static_scratch_ptr(&ws) != hipSuccess) return UMEM_ERR_HIP;
  return forward_into(desc, T, q_row, q_col, k_row, k_col, core, values, perm, w_proj, w_out, out,
                      idx_out, w_out_scores, ws, UMEM_STATIC_SCRATCH_BYTES, stream);
}

UMEM_API const char* umem_status_string(umem_status status) {
  switch (status) {
    case UMEM_OK: return "ok";
    case UMEM_ERR_INVALID_ARG: return "invalid argument";
    case UMEM_ERR_UNSUPPORTED: return "unsupported by this library";
    case UMEM_ERR_WORKSPACE: return "workspace too small or misaligned";
    case UMEM_ERR_HIP: return "HIP launch error";
    case UMEM_ERR_SCRATCH_LIMIT: return "needs more scratch than the static buffer holds";
  }
  return "unknown status";
}

}  // extern "C"
