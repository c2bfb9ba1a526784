// C ABI of the operators around the linear layers (token tables, group norm,
// one norm over many tensors): argument checks and dispatch. The operations and
// their conventions are specified in include/dpsgd.h.
#include <math.h>

#include "common.h"

namespace dpsgd {
namespace {

constexpr int64_t kI32Max = 0x7FFFFFFF;
constexpr int64_t kMostEntries = INT64_C(1) << 40;   // of one tensor

bool valid_dtype(int32_t d) { return d == DPSGD_F32 || d == DPSGD_BF16; }
bool aligned(const void* p, size_t n) { return p && reinterpret_cast<uintptr_t>(p) % n == 0; }

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const char *p = static_cast<const char*>(a), *q = static_cast<const char*>(b);
  return p && q && p < q + nb && q < p + na;
}

int check_embedding(const dpsgd_embedding* e, bool data) {
  if (!e) return DPSGD_ERR_INVALID_ARG;
  if (e->index_dtype != DPSGD_I32 && e->index_dtype != DPSGD_I64) return DPSGD_ERR_UNSUPPORTED;
  if (e->B < 1 || e->T < 1 || e->n_rows < 1 || e->d < 1) return DPSGD_ERR_INVALID_ARG;
  if (e->B > (INT64_C(1) << 30) || e->T > (INT64_C(1) << 30) / e->B || e->n_rows > kI32Max)
    return DPSGD_ERR_INVALID_ARG;
  if (e->d > (INT64_C(1) << 20) || e->d > kMostEntries / (e->B * e->T) ||
      e->d > kMostEntries / e->n_rows)
    return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(e->scale)) return DPSGD_ERR_INVALID_ARG;
  if (data && !aligned(e->ids, e->index_dtype == DPSGD_I64 ? 8 : 4)) return DPSGD_ERR_INVALID_ARG;
  return DPSGD_OK;
}

int check_group_norm(const dpsgd_group_norm* n) {
  if (!n) return DPSGD_ERR_INVALID_ARG;
  if (!valid_dtype(n->dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (n->act < DPSGD_ACT_NONE || n->act > DPSGD_ACT_GELU) return DPSGD_ERR_UNSUPPORTED;
  if (n->B < 1 || n->S < 1 || n->C < 1 || n->groups < 1) return DPSGD_ERR_INVALID_ARG;
  if (n->B > kI32Max || n->S > kI32Max / n->B || n->C > (INT64_C(1) << 20)) return DPSGD_ERR_INVALID_ARG;
  if (n->C > kMostEntries / (n->B * n->S)) return DPSGD_ERR_INVALID_ARG;
  if (n->groups > n->C || n->C % n->groups != 0) return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(n->eps) || !(n->eps > 0.0f)) return DPSGD_ERR_INVALID_ARG;
  return DPSGD_OK;
}

int check_affine(const dpsgd_group_norm* n) {
  if (n->gamma && !aligned(n->gamma, 4)) return DPSGD_ERR_INVALID_ARG;
  if (n->beta && !aligned(n->beta, 4)) return DPSGD_ERR_INVALID_ARG;
  return DPSGD_OK;
}

int check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return DPSGD_ERR_WORKSPACE;
  return aligned16(ws) ? DPSGD_OK : DPSGD_ERR_INVALID_ARG;
}

int check_tensors(const dpsgd_layer* layers, int32_t n) {
  if (!layers || n < 1) return DPSGD_ERR_INVALID_ARG;
  for (int32_t l = 0; l < n; ++l) {
    const dpsgd_layer& L = layers[l];
    if (L.d_in < 1 || L.d_out < 1 || L.d_in > kI32Max || L.d_out > kI32Max ||
        L.d_out > kMostEntries / L.d_in)
      return DPSGD_ERR_INVALID_ARG;
  }
  return DPSGD_OK;
}

}  // namespace
}  // namespace dpsgd

using namespace dpsgd;

extern "C" {

int dpsgd_embedding_lookup(const dpsgd_embedding* emb, const void* table, int32_t table_dtype,
                           void* out, int32_t out_dtype, void* stream) {
  const int st = check_embedding(emb, true);
  if (st != DPSGD_OK) return st;
  if (!valid_dtype(table_dtype) || !valid_dtype(out_dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (!aligned(table, 16) || !aligned(out, 16)) return DPSGD_ERR_INVALID_ARG;
  return launch_embedding_lookup(*emb, table, table_dtype, out, out_dtype,
                                 static_cast<hipStream_t>(stream));
}

size_t dpsgd_embedding_workspace_bytes(const dpsgd_embedding* emb) {
  if (check_embedding(emb, false) != DPSGD_OK) return 0;
  return embedding_workspace_bytes(*emb);
}

int dpsgd_embedding_norms(const dpsgd_embedding* emb, const void* G, int32_t dtype,
                          float* norms_sq, int32_t accumulate, void* workspace,
                          size_t workspace_bytes, void* stream) {
  int st = check_embedding(emb, true);
  if (st != DPSGD_OK) return st;
  if (!valid_dtype(dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (!aligned(G, 16) || !aligned(norms_sq, 4)) return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, embedding_workspace_bytes(*emb));
  if (st != DPSGD_OK) return st;
  return launch_embedding_norms(*emb, G, dtype, norms_sq, accumulate ? 1 : 0, workspace,
                                static_cast<hipStream_t>(stream));
}

int dpsgd_embedding_clip_accumulate(const dpsgd_embedding* emb, const void* G, int32_t dtype,
                                    const float* norms_sq, float C, float* grad,
                                    int32_t accumulate, float* factors_out, uint8_t* mask_out,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_embedding(emb, true);
  if (st != DPSGD_OK) return st;
  if (!valid_dtype(dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (!aligned(G, 16) || !aligned(grad, 16)) return DPSGD_ERR_INVALID_ARG;
  if (norms_sq) {
    if (!aligned(norms_sq, 4) || !(C > 0.0f)) return DPSGD_ERR_INVALID_ARG;   // NaN too
    if (factors_out && !aligned(factors_out, 4)) return DPSGD_ERR_INVALID_ARG;
    // The factors are formed from the norms while they, and grad, are written.
    const size_t n = (size_t)emb->B * sizeof(float);
    const size_t ng = (size_t)(emb->n_rows * emb->d) * sizeof(float);
    if (overlaps(norms_sq, n, grad, ng) || overlaps(norms_sq, n, factors_out, n) ||
        overlaps(norms_sq, n, mask_out, (size_t)emb->B) || overlaps(grad, ng, factors_out, n) ||
        overlaps(grad, ng, mask_out, (size_t)emb->B))
      return DPSGD_ERR_INVALID_ARG;
  } else if (factors_out || mask_out) {
    return DPSGD_ERR_INVALID_ARG;
  }
  st = check_workspace(workspace, workspace_bytes, embedding_workspace_bytes(*emb));
  if (st != DPSGD_OK) return st;
  return launch_embedding_sum(*emb, G, dtype, norms_sq, C, grad, accumulate ? 1 : 0, factors_out,
                              mask_out, workspace, static_cast<hipStream_t>(stream));
}

size_t dpsgd_group_norm_workspace_bytes(const dpsgd_group_norm* gn) {
  if (check_group_norm(gn) != DPSGD_OK) return 0;
  return group_norm_workspace_bytes(*gn);
}

int dpsgd_group_norm_forward(const dpsgd_group_norm* gn, const void* x, void* y, float* mean,
                             float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_group_norm(gn);
  if (st == DPSGD_OK) st = check_affine(gn);
  if (st != DPSGD_OK) return st;
  if (!aligned(x, 16) || !aligned(y, 16)) return DPSGD_ERR_INVALID_ARG;
  if ((mean && !aligned(mean, 4)) || (rstd && !aligned(rstd, 4))) return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, group_norm_workspace_bytes(*gn));
  if (st != DPSGD_OK) return st;
  return launch_group_norm_forward(*gn, x, y, mean, rstd, workspace,
                                   static_cast<hipStream_t>(stream));
}

int dpsgd_group_norm_backward(const dpsgd_group_norm* gn, const void* x, const void* dy,
                              const float* mean, const float* rstd, void* dx, float* dgamma,
                              float* dbeta, void* workspace, size_t workspace_bytes,
                              void* stream) {
  int st = check_group_norm(gn);
  if (st == DPSGD_OK) st = check_affine(gn);
  if (st != DPSGD_OK) return st;
  if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16) || dx == x) return DPSGD_ERR_INVALID_ARG;
  if (!aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, group_norm_workspace_bytes(*gn));
  if (st != DPSGD_OK) return st;
  return launch_group_norm_backward(*gn, x, dy, mean, rstd, dx, dgamma, dbeta, workspace,
                                    static_cast<hipStream_t>(stream));
}

size_t dpsgd_global_norm_workspace_bytes(const dpsgd_layer* layers, int32_t n_layers) {
  if (check_tensors(layers, n_layers) != DPSGD_OK) return 0;
  return global_norm_workspace_bytes(layers, n_layers);
}

int dpsgd_global_norm_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* grads, float* norm_out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  int st = check_tensors(layers, n_layers);
  if (st != DPSGD_OK) return st;
  if (!grads || !aligned(norm_out, 4)) return DPSGD_ERR_INVALID_ARG;
  for (int32_t l = 0; l < n_layers; ++l)
    if (!aligned(grads[l], 16)) return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, global_norm_workspace_bytes(layers, n_layers));
  if (st != DPSGD_OK) return st;
  return launch_global_clip(layers, n_layers, grads, nullptr, INFINITY, norm_out, nullptr,
                            workspace, static_cast<hipStream_t>(stream));
}

int dpsgd_global_clip_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* grads, float* const* outs, float max_norm,
                            float* norm_out, float* factor_out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  int st = check_tensors(layers, n_layers);
  if (st != DPSGD_OK) return st;
  if (!grads || !outs || !(max_norm > 0.0f)) return DPSGD_ERR_INVALID_ARG;
  if ((norm_out && !aligned(norm_out, 4)) || (factor_out && !aligned(factor_out, 4)))
    return DPSGD_ERR_INVALID_ARG;
  for (int32_t l = 0; l < n_layers; ++l)
    if (!aligned(grads[l], 16) || !aligned(outs[l], 16)) return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, global_norm_workspace_bytes(layers, n_layers));
  if (st != DPSGD_OK) return st;
  return launch_global_clip(layers, n_layers, grads, outs, max_norm, norm_out, factor_out,
                            workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
