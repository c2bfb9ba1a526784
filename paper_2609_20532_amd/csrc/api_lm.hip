// C ABI of the operators between and behind a model's blocks (log probabilities and
// loss, residual norms, AdamW with 8-bit moments): argument checks and dispatch. The
// operations and their conventions are specified in include/dpsgd.h.
#include <math.h>

#include "common.h"

namespace dpsgd {
namespace {

constexpr int64_t kI32Max = 0x7FFFFFFF;
constexpr int64_t kMostEntries = INT64_C(1) << 40;   // of one tensor
constexpr int64_t kMostStride = INT64_C(1) << 31;

bool valid_dtype(int32_t d) { return d == DPSGD_F32 || d == DPSGD_BF16; }
size_t element(int32_t dtype) { return dtype == DPSGD_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t n) { return p && reinterpret_cast<uintptr_t>(p) % n == 0; }
bool may_aligned(const void* p, size_t n) { return !p || aligned(p, n); }

int check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws || have < need) return DPSGD_ERR_WORKSPACE;
  return aligned16(ws) ? DPSGD_OK : DPSGD_ERR_INVALID_ARG;
}

// Memory that a call reads or writes. A written range overlaps no other one, except
// one that it is named to be equal to (`same`: the index of that range, or -1).
struct Range {
  const void* p;
  size_t bytes;
  bool written;
  int same;
};

bool apart(const Range* r, int n) {
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < i; ++j) {
      if (!r[i].p || !r[j].p || !(r[i].written || r[j].written)) continue;
      const char *p = static_cast<const char*>(r[i].p), *q = static_cast<const char*>(r[j].p);
      if (p >= q + r[j].bytes || q >= p + r[i].bytes) continue;
      if (p == q && (r[i].same == j || r[j].same == i)) continue;
      return false;
    }
  }
  return true;
}

int check_logits(const dpsgd_logits* d, bool data) {
  if (!d) return DPSGD_ERR_INVALID_ARG;
  if (!valid_dtype(d->dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (d->index_dtype != DPSGD_I32 && d->index_dtype != DPSGD_I64) return DPSGD_ERR_UNSUPPORTED;
  if (d->B < 1 || d->T < 1 || d->V < 1 || d->V > (INT64_C(1) << 24)) return DPSGD_ERR_INVALID_ARG;
  if (d->B > (INT64_C(1) << 30) || d->T > (INT64_C(1) << 30) / d->B) return DPSGD_ERR_INVALID_ARG;
  if (d->stride < d->V || d->stride > kMostStride || d->stride > kMostEntries / (d->B * d->T))
    return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(d->scale) || !(d->scale > 0.0f)) return DPSGD_ERR_INVALID_ARG;
  if (data && !may_aligned(d->targets, d->index_dtype == DPSGD_I64 ? 8 : 4))
    return DPSGD_ERR_INVALID_ARG;
  return DPSGD_OK;
}

Range targets_of(const dpsgd_logits* d) {
  return {d->targets, (size_t)(d->B * d->T) * (d->index_dtype == DPSGD_I64 ? 8 : 4), false, -1};
}

// The rows from the first entry of the first to the last entry of the last.
Range rows_of(const dpsgd_logits* d, const void* p, int64_t stride, bool written, int same) {
  return {p, (size_t)((d->B * d->T - 1) * stride + d->V) * element(d->dtype), written, same};
}

Range per_row(const dpsgd_logits* d, const void* p, size_t bytes, bool written) {
  return {p, (size_t)(d->B * d->T) * bytes, written, -1};
}

bool valid_gradient(const dpsgd_logits* d, const void* logits, const void* dlogits, int64_t stride) {
  if (!aligned(logits, element(d->dtype)) || !aligned(dlogits, element(d->dtype))) return false;
  if (stride < d->V || stride > kMostStride || stride > kMostEntries / (d->B * d->T)) return false;
  return dlogits != logits || stride == d->stride;
}

int check_residual_norm(const dpsgd_residual_norm* n) {
  if (!n) return DPSGD_ERR_INVALID_ARG;
  if (!valid_dtype(n->dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (n->kind != DPSGD_ROW_NORM_LAYER && n->kind != DPSGD_ROW_NORM_RMS) return DPSGD_ERR_UNSUPPORTED;
  if (n->B < 1 || n->S < 1 || n->B > kI32Max || n->S > kI32Max / n->B) return DPSGD_ERR_INVALID_ARG;
  if (n->C < 1 || n->C > 16384) return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(n->eps) || !(n->eps > 0.0f) || !isfinite(n->residual_scale)) return DPSGD_ERR_INVALID_ARG;
  return DPSGD_OK;
}

// The descriptor's pointers, and what a call without a block may not have.
int check_affine(const dpsgd_residual_norm* n, const void* block) {
  const float* const ps[5] = {n->gamma, n->beta, n->post_gamma, n->post_beta, n->gate};
  for (const float* p : ps)
    if (!may_aligned(p, 16)) return DPSGD_ERR_INVALID_ARG;
  if (!n->post && (n->post_gamma || n->post_beta)) return DPSGD_ERR_INVALID_ARG;
  if (!block && (n->post || n->gate)) return DPSGD_ERR_INVALID_ARG;
  return DPSGD_OK;
}

constexpr int kAffine = 5;

void affine_ranges(const dpsgd_residual_norm* n, Range* to) {
  const size_t c = (size_t)n->C * sizeof(float);
  to[0] = {n->gamma, c, false, -1};
  to[1] = {n->beta, c, false, -1};
  to[2] = {n->post_gamma, c, false, -1};
  to[3] = {n->post_beta, c, false, -1};
  to[4] = {n->gate, n->gate_per_example ? c * (size_t)n->B : c, false, -1};
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

bool distinct_ids(const dpsgd_layer* layers, int32_t n) {
  for (int32_t i = 0; i < n; ++i)
    for (int32_t j = 0; j < i; ++j)
      if (layers[i].tensor_id == layers[j].tensor_id) return false;
  return true;
}

}  // namespace
}  // namespace dpsgd

using namespace dpsgd;

extern "C" {

size_t dpsgd_token_workspace_bytes(const dpsgd_logits* desc, int32_t k) {
  if (check_logits(desc, false) != DPSGD_OK || k < 0 || k > DPSGD_MOST_ALTERNATIVES) return 0;
  return token_workspace_bytes(*desc, k);
}

int dpsgd_token_logprobs(const dpsgd_logits* desc, const void* logits, float* logprobs, float* lse,
                         float* entropy, int32_t k, int64_t* top_ids, float* top_logprobs,
                         void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_logits(desc, true);
  if (st != DPSGD_OK) return st;
  if (!aligned(logits, element(desc->dtype))) return DPSGD_ERR_INVALID_ARG;
  if (k < 0 || k > DPSGD_MOST_ALTERNATIVES) return DPSGD_ERR_INVALID_ARG;
  if (k == 0 ? (top_ids || top_logprobs) : !(top_ids || top_logprobs)) return DPSGD_ERR_INVALID_ARG;
  if (!logprobs && !lse && !entropy && k == 0) return DPSGD_ERR_INVALID_ARG;
  if (logprobs && !desc->targets) return DPSGD_ERR_INVALID_ARG;
  if (!may_aligned(logprobs, 4) || !may_aligned(lse, 4) || !may_aligned(entropy, 4) ||
      !may_aligned(top_ids, 8) || !may_aligned(top_logprobs, 4))
    return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, token_workspace_bytes(*desc, k));
  if (st != DPSGD_OK) return st;
  const Range r[] = {rows_of(desc, logits, desc->stride, false, -1), targets_of(desc),
                     per_row(desc, logprobs, 4, true), per_row(desc, lse, 4, true),
                     per_row(desc, entropy, 4, true), per_row(desc, top_ids, 8 * (size_t)k, true),
                     per_row(desc, top_logprobs, 4 * (size_t)k, true),
                     {workspace, token_workspace_bytes(*desc, k), true, -1}};
  if (!apart(r, 8)) return DPSGD_ERR_INVALID_ARG;
  return launch_token_logprobs(*desc, logits, logprobs, lse, entropy, k, top_ids, top_logprobs,
                               workspace, static_cast<hipStream_t>(stream));
}

int dpsgd_token_logprobs_backward(const dpsgd_logits* desc, const void* logits, const float* lse,
                                  const float* entropy, const float* grad_logprobs,
                                  const float* grad_lse, const float* grad_entropy, void* dlogits,
                                  int64_t dlogits_stride, void* stream) {
  const int st = check_logits(desc, true);
  if (st != DPSGD_OK) return st;
  if (!valid_gradient(desc, logits, dlogits, dlogits_stride)) return DPSGD_ERR_INVALID_ARG;
  if (!grad_logprobs && !grad_lse && !grad_entropy) return DPSGD_ERR_INVALID_ARG;
  if (grad_logprobs && !desc->targets) return DPSGD_ERR_INVALID_ARG;
  if (!aligned(lse, 4) || (grad_entropy && !entropy)) return DPSGD_ERR_INVALID_ARG;
  if (!may_aligned(entropy, 4) || !may_aligned(grad_logprobs, 4) || !may_aligned(grad_lse, 4) ||
      !may_aligned(grad_entropy, 4))
    return DPSGD_ERR_INVALID_ARG;
  const Range r[] = {rows_of(desc, logits, desc->stride, false, -1), targets_of(desc),
                     per_row(desc, lse, 4, false), per_row(desc, entropy, 4, false),
                     per_row(desc, grad_logprobs, 4, false), per_row(desc, grad_lse, 4, false),
                     per_row(desc, grad_entropy, 4, false),
                     rows_of(desc, dlogits, dlogits_stride, true, 0)};
  if (!apart(r, 8)) return DPSGD_ERR_INVALID_ARG;
  return launch_token_backward(*desc, logits, lse, entropy, grad_logprobs, grad_lse, grad_entropy,
                               dlogits, dlogits_stride, static_cast<hipStream_t>(stream));
}

int dpsgd_token_loss(const dpsgd_logits* desc, const void* logits, const float* weights,
                     float* losses, float* logprobs, void* dlogits, int64_t dlogits_stride,
                     void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_logits(desc, true);
  if (st != DPSGD_OK) return st;
  if (!desc->targets || !valid_gradient(desc, logits, dlogits, dlogits_stride))
    return DPSGD_ERR_INVALID_ARG;
  if (!may_aligned(weights, 4) || !may_aligned(losses, 4) || !may_aligned(logprobs, 4))
    return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, token_workspace_bytes(*desc, 0));
  if (st != DPSGD_OK) return st;
  const Range r[] = {rows_of(desc, logits, desc->stride, false, -1), targets_of(desc),
                     per_row(desc, weights, 4, false),
                     {losses, (size_t)desc->B * 4, true, -1}, per_row(desc, logprobs, 4, true),
                     rows_of(desc, dlogits, dlogits_stride, true, 0),
                     {workspace, token_workspace_bytes(*desc, 0), true, -1}};
  if (!apart(r, 7)) return DPSGD_ERR_INVALID_ARG;
  return launch_token_loss(*desc, logits, weights, losses, logprobs, dlogits, dlogits_stride,
                           workspace, static_cast<hipStream_t>(stream));
}

int dpsgd_residual_norm_forward(const dpsgd_residual_norm* desc, const void* x, const void* block,
                                void* r, void* y, float* stats, void* stream) {
  int st = check_residual_norm(desc);
  if (st == DPSGD_OK) st = check_affine(desc, block);
  if (st != DPSGD_OK) return st;
  if (!aligned(x, 16) || !aligned(y, 16)) return DPSGD_ERR_INVALID_ARG;
  if (!may_aligned(block, 16) || !may_aligned(r, 16) || !may_aligned(stats, 16))
    return DPSGD_ERR_INVALID_ARG;
  const size_t rows = (size_t)(desc->B * desc->S), n = rows * (size_t)desc->C * element(desc->dtype);
  Range ranges[5 + kAffine] = {{x, n, false, 2}, {block, n, false, 3}, {r, n, true, 0},
                               {y, n, true, 1}, {stats, rows * 16, true, -1}};
  affine_ranges(desc, ranges + 5);
  if (!apart(ranges, 5 + kAffine)) return DPSGD_ERR_INVALID_ARG;
  return launch_residual_norm_forward(*desc, x, block, r, y, stats,
                                      static_cast<hipStream_t>(stream));
}

size_t dpsgd_residual_norm_workspace_bytes(const dpsgd_residual_norm* desc) {
  if (check_residual_norm(desc) != DPSGD_OK) return 0;
  return residual_norm_workspace_bytes(*desc);
}

int dpsgd_residual_norm_backward(const dpsgd_residual_norm* desc, const void* block, const void* r,
                                 const void* dy, const void* dr, const float* stats, void* dx,
                                 void* dblock, float* dgamma, float* dbeta, float* dgate,
                                 float* dpost_gamma, float* dpost_beta, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  int st = check_residual_norm(desc);
  if (st == DPSGD_OK) st = check_affine(desc, block);
  if (st != DPSGD_OK) return st;
  if (!aligned(r, 16) || !aligned(dy, 16) || !aligned(stats, 16)) return DPSGD_ERR_INVALID_ARG;
  if (!may_aligned(block, 16) || !may_aligned(dr, 16) || !may_aligned(dx, 16) || !may_aligned(dblock, 16))
    return DPSGD_ERR_INVALID_ARG;
  if (!block != !dblock || (!block && dgate) || (!desc->post && (dpost_gamma || dpost_beta)))
    return DPSGD_ERR_INVALID_ARG;
  float* const grads[kAffine] = {dgamma, dbeta, dgate, dpost_gamma, dpost_beta};
  bool any = dx || dblock;
  for (const float* g : grads) {
    if (!may_aligned(g, 16)) return DPSGD_ERR_INVALID_ARG;
    any = any || g;
  }
  if (!any) return DPSGD_ERR_INVALID_ARG;
  st = check_workspace(workspace, workspace_bytes, residual_norm_workspace_bytes(*desc));
  if (st != DPSGD_OK) return st;
  const size_t rows = (size_t)(desc->B * desc->S), n = rows * (size_t)desc->C * element(desc->dtype);
  const size_t ng = (size_t)(desc->B * desc->C) * sizeof(float);
  Range ranges[8 + 2 * kAffine] = {{block, n, false, -1}, {r, n, false, -1}, {dy, n, false, 6},
                                   {dr, n, false, 5}, {stats, rows * 16, false, -1},
                                   {dx, n, true, 3}, {dblock, n, true, 2},
                                   {workspace, residual_norm_workspace_bytes(*desc), true, -1}};
  affine_ranges(desc, ranges + 8);
  for (int k = 0; k < kAffine; ++k) ranges[8 + kAffine + k] = {grads[k], ng, true, -1};
  if (!apart(ranges, 8 + 2 * kAffine)) return DPSGD_ERR_INVALID_ARG;
  return launch_residual_norm_backward(*desc, block, r, dy, dr, stats, dx, dblock, grads, workspace,
                                       static_cast<hipStream_t>(stream));
}

int dpsgd_noise_adamw8_multi(const dpsgd_layer* layers, int32_t n_layers,
                             const float* const* grads, float* const* params,
                             uint8_t* const* exp_avgs, uint8_t* const* exp_avg_sqs,
                             uint8_t* const* exponents, float* const* noisy_outs, float sigma,
                             float C, uint64_t seed, uint32_t step, float scale,
                             const dpsgd_adamw* opt, int32_t rounding, uint64_t round_seed,
                             void* stream) {
  const int st = check_tensors(layers, n_layers);
  if (st != DPSGD_OK) return st;
  if (rounding != DPSGD_ROUND_NEAREST && rounding != DPSGD_ROUND_STOCHASTIC)
    return DPSGD_ERR_UNSUPPORTED;
  if (!grads || !params || !exp_avgs || !exp_avg_sqs || !exponents || !opt)
    return DPSGD_ERR_INVALID_ARG;
  for (int32_t l = 0; l < n_layers; ++l) {
    const void* need[5] = {grads[l], params[l], exp_avgs[l], exp_avg_sqs[l], exponents[l]};
    for (const void* p : need)
      if (!aligned(p, 16)) return DPSGD_ERR_INVALID_ARG;
    if (noisy_outs && !may_aligned(noisy_outs[l], 16)) return DPSGD_ERR_INVALID_ARG;
  }
  if (!(sigma >= 0.0f) || isinf(sigma)) return DPSGD_ERR_INVALID_ARG;   // NaN too
  if (!(C > 0.0f) || isinf(C)) return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(scale)) return DPSGD_ERR_INVALID_ARG;
  const dpsgd_adamw& o = *opt;
  if (!isfinite(o.lr) || o.lr < 0.0f) return DPSGD_ERR_INVALID_ARG;
  if (!(o.beta1 >= 0.0f && o.beta1 < 1.0f) || !(o.beta2 >= 0.0f && o.beta2 < 1.0f))
    return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(o.eps) || !(o.eps > 0.0f)) return DPSGD_ERR_INVALID_ARG;
  if (!isfinite(o.weight_decay) || o.weight_decay < 0.0f) return DPSGD_ERR_INVALID_ARG;
  if (o.t == 0) return DPSGD_ERR_INVALID_ARG;
  if (!distinct_ids(layers, n_layers)) return DPSGD_ERR_INVALID_ARG;
  return launch_noise_adamw8(layers, n_layers, grads, params, exp_avgs, exp_avg_sqs, exponents,
                             noisy_outs, sigma, C, seed, step, scale, o, rounding, round_seed,
                             static_cast<hipStream_t>(stream));
}

int dpsgd_adamw8_pack_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* exp_avgs_in, const float* const* exp_avg_sqs_in,
                            uint8_t* const* exp_avgs, uint8_t* const* exp_avg_sqs,
                            uint8_t* const* exponents, void* stream) {
  const int st = check_tensors(layers, n_layers);
  if (st != DPSGD_OK) return st;
  if (!exp_avgs_in || !exp_avg_sqs_in || !exp_avgs || !exp_avg_sqs || !exponents)
    return DPSGD_ERR_INVALID_ARG;
  for (int32_t l = 0; l < n_layers; ++l) {
    const void* need[5] = {exp_avgs_in[l], exp_avg_sqs_in[l], exp_avgs[l], exp_avg_sqs[l], exponents[l]};
    for (const void* p : need)
      if (!aligned(p, 16)) return DPSGD_ERR_INVALID_ARG;
  }
  return launch_adamw8_pack(layers, n_layers, exp_avgs_in, exp_avg_sqs_in, exp_avgs, exp_avg_sqs,
                            exponents, static_cast<hipStream_t>(stream));
}

int dpsgd_adamw8_unpack_multi(const dpsgd_layer* layers, int32_t n_layers,
                              const uint8_t* const* exp_avgs, const uint8_t* const* exp_avg_sqs,
                              const uint8_t* const* exponents, void* const* exp_avgs_out,
                              void* const* exp_avg_sqs_out, int32_t out_dtype, void* stream) {
  const int st = check_tensors(layers, n_layers);
  if (st != DPSGD_OK) return st;
  if (!valid_dtype(out_dtype)) return DPSGD_ERR_UNSUPPORTED;
  if (!exp_avgs || !exp_avg_sqs || !exponents || !exp_avgs_out || !exp_avg_sqs_out)
    return DPSGD_ERR_INVALID_ARG;
  for (int32_t l = 0; l < n_layers; ++l) {
    const void* need[5] = {exp_avgs[l], exp_avg_sqs[l], exponents[l], exp_avgs_out[l], exp_avg_sqs_out[l]};
    for (const void* p : need)
      if (!aligned(p, 16)) return DPSGD_ERR_INVALID_ARG;
  }
  return launch_adamw8_unpack(layers, n_layers, exp_avgs, exp_avg_sqs, exponents, exp_avgs_out,
                              exp_avg_sqs_out, out_dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"
