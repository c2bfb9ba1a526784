/*
 * dpsgd.h -- C ABI of the MI355X (gfx950) DP-SGD gradient-step library.
 *
 * The library computes, on one GPU, the part of a DP-SGD step that the
 * paper's protocol gives to the untrusted GPU (the algorithm "GPU-side
 * Gradient Computation and Local Update" and Section 2.2, "DP-SGD"):
 *
 *   per-example gradient of each linear layer   g_i = G_i^T A_i
 *   per-example L2 norm over all layers        n_i = sqrt(sum_l ||g_{i,l}||_F^2)
 *   clip factor                                 c_i = min(1, C / n_i)
 *   clipped sum over the batch                  S_l = sum_i c_i g_{i,l}
 *   Gaussian noise of scale sigma*C             out = scale * (S_l + sigma*C*z)
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - A linear layer y_t = W x_t is described by a dpsgd_layer: the
 *    activations A [B][T][d_in] and output gradients G [B][T][d_out]
 *    (G[i][t] = dloss_i/dy_t), both row-major and contiguous, both of the
 *    same element type (float32 or bfloat16).
 *  - Gradient-shaped buffers are float32 [d_out][d_in], row-major (the layout
 *    of W itself).
 *  - Every pointer to tensor data is a DEVICE pointer owned by the caller.
 *    The library allocates no device memory, keeps no pointer after a call
 *    returns and holds no mutable global state; calls are thread-safe. The
 *    one exception is dpsgd_per_example_norms_multi_noalloc, whose scratch
 *    array lives in each GPU's memory (see there).
 *  - Arrays of descriptors (dpsgd_layer*, float* const*) are HOST memory and
 *    are read before the call returns.
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *    Every call only enqueues kernels on it and returns; results are valid
 *    once the caller synchronises with the stream. Faults inside a kernel
 *    surface at that synchronisation.
 *  - Every entry point returns a dpsgd_status. Nothing aborts or throws across
 *    the ABI. An error found by the argument checks returns before anything
 *    is enqueued. DPSGD_ERR_HIP (a launch the runtime rejected) and
 *    DPSGD_ERR_INVALID_ARG for a grid too large for one launch (beyond 2^31
 *    workgroups, far past any size the checks accept in practice) can come
 *    after earlier kernels of the same call were enqueued; the outputs are
 *    then unspecified.
 *  - Results are deterministic: the same inputs on the same device give
 *    bitwise-identical outputs (no floating-point atomics).
 *  - Arithmetic: products of bf16 inputs are exact in float32 and all sums
 *    accumulate in float32.
 */
#ifndef DPSGD_H_
#define DPSGD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dpsgd_dtype {
  DPSGD_F32 = 0,   /* IEEE binary32                               */
  DPSGD_BF16 = 1   /* bfloat16 (upper 16 bits of a binary32)       */
} dpsgd_dtype;

typedef enum dpsgd_norm_mode {
  DPSGD_NORM_AUTO = 0,         /* pick per layer by arithmetic cost           */
  DPSGD_NORM_GHOST = 1,        /* Gram form: sum_{t,s} (a_t.a_s)(g_t.g_s)     */
  DPSGD_NORM_MATERIALIZE = 2,  /* ||G_i^T A_i||_F^2, tile kept in registers   */
  DPSGD_NORM_CLOSED_FORM = 3   /* T = 1: ||a_i||^2 ||g_i||^2. Only reported by
                                  dpsgd_select_norm_mode; not accepted as a
                                  mode argument (DPSGD_ERR_UNSUPPORTED)       */
} dpsgd_norm_mode;

typedef enum dpsgd_status {
  DPSGD_OK = 0,
  DPSGD_ERR_INVALID_ARG = -1,  /* null or misaligned required pointer, size < 1 or overflow, C <= 0 or NaN,
                                  sigma < 0 or NaN, scale not finite                      */
  DPSGD_ERR_UNSUPPORTED = -2,  /* unknown dtype or mode, mixed dtypes in one call         */
  DPSGD_ERR_WORKSPACE = -3,    /* workspace NULL or smaller than the *_workspace_bytes value */
  DPSGD_ERR_HIP = -4           /* the HIP runtime rejected a launch                       */
} dpsgd_status;

/* One linear layer y = x W^T (W: [d_out][d_in]) as seen by one batch.
 * Paper: Section 2.2, per-example gradient of the trainable parameters. */
typedef struct dpsgd_layer {
  const void* A;       /* [B][T][d_in]  activations, dtype; 16-byte aligned      */
  const void* G;       /* [B][T][d_out] output gradients dloss_i/dy_t, dtype;
                          16-byte aligned                                         */
  int64_t B;           /* examples in the batch, >= 1                            */
  int64_t T;           /* positions per example (sequence length), >= 1          */
  int64_t d_in;        /* >= 1                                                   */
  int64_t d_out;       /* >= 1                                                   */
  int32_t dtype;       /* dpsgd_dtype, shared by A and G                         */
  uint32_t tensor_id;  /* third Philox counter word of this layer's noise; the
                          layers of one noise call must have distinct ids     */
} dpsgd_layer;

/* ---------------------------------------------------------------------------
 * Per-example norms.  Paper: Section 2.2 (per-example clipping uses
 * ||g_t(x_i)||_2 over all trainable parameters); GPU-side algorithm, clip step.
 *
 * norms_sq[i] = (accumulate ? norms_sq[i] : 0) + sum_l ||G_{l,i}^T A_{l,i}||_F^2
 *
 * over the n_layers layers of the call, all with the same B. One call over all
 * layers of a step gives the squared global norm; per-layer calls with
 * accumulate=1 give the same value up to float32 summation order.
 *   mode      dpsgd_norm_mode, applied to every layer (AUTO picks per layer).
 *   norms_sq  float32 [B], device.
 *   workspace device scratch of at least dpsgd_norms_workspace_bytes(...)
 *             bytes, 16-byte aligned (DPSGD_ERR_INVALID_ARG otherwise); its
 *             contents on entry do not matter and are clobbered. It holds
 *             per-example partials and, when a bf16 layer with T > 256 and
 *             widths that are multiples of 64 runs the Gram form, a park
 *             area of at most 128 MB (256 KB per workgroup of that kernel,
 *             or, when few tiles are split along the columns, two 256 KB
 *             partial tiles per part), or, when the Gram-form layers have few
 *             tiles in all, at most 112 partial tiles of 64 KB.
 * T = 1 layers always use the closed form ||a||^2 ||g||^2 whatever the mode.
 * ------------------------------------------------------------------------- */
size_t dpsgd_norms_workspace_bytes(const dpsgd_layer* layers, int32_t n_layers, int32_t mode);

/* The form that dpsgd_per_example_norms[_multi] runs for this layer under
 * DPSGD_NORM_AUTO: DPSGD_NORM_CLOSED_FORM for T = 1 (under every mode),
 * otherwise DPSGD_NORM_GHOST or DPSGD_NORM_MATERIALIZE; or a negative
 * dpsgd_status for an invalid descriptor. (In dpsgd_clipped_sum_multi a
 * layer with a narrow side may take the stored form instead; see there. In a
 * call of several layers one near the line may take the form of the others,
 * and in a call whose partials together exceed DPSGD_NOALLOC_SCRATCH_BYTES a
 * layer reported as materialised may run the Gram form.) */
int32_t dpsgd_select_norm_mode(const dpsgd_layer* layer);

int dpsgd_per_example_norms(const dpsgd_layer* layer, int32_t mode, float* norms_sq,
                            int32_t accumulate, void* workspace, size_t workspace_bytes,
                            void* stream);

int dpsgd_per_example_norms_multi(const dpsgd_layer* layers, int32_t n_layers, int32_t mode,
                                  float* norms_sq, int32_t accumulate, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Per-example norms with no workspace argument, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation.
 *
 * The operation, arguments and results of dpsgd_per_example_norms_multi,
 * with the per-example partials kept in a scratch array of
 * DPSGD_NOALLOC_SCRATCH_BYTES bytes that the library holds in the memory of
 * each GPU it runs on, from the first call on that GPU until the process
 * ends. The call allocates nothing. Results equal the workspace call's bit
 * for bit (the same kernels run), except for bf16 Gram-form layers with
 * T > 256: the workspace call runs them on 256-row tiles, whose park area
 * the array does not hold, this call on 128-row tiles, so their norms agree
 * to float32 rounding.
 *  - Runs on the current device (hipSetDevice), whose stream `stream` must be.
 *    The first call on a device resolves the array's address there (no
 *    stream work); make it before capturing a graph that contains the call.
 *  - DPSGD_ERR_WORKSPACE when the layers need more partial storage than the
 *    array holds (about 2M float partials: B times the sum over layers of
 *    the partials per example, a T > 256 Gram-form layer counting its
 *    128-row tile pairs); checked before anything else touches the device. DPSGD_ERR_HIP when the runtime cannot give the
 *    array's address on the current device. Other errors as in
 *    dpsgd_per_example_norms_multi.
 *  - Every call on one GPU uses that GPU's one array, which keeps the last
 *    call's partials: calls that overlap in time on one GPU (different
 *    streams, or host threads without ordering between them) race, and
 *    their results are undefined.
 * ------------------------------------------------------------------------- */
#define DPSGD_NOALLOC_SCRATCH_BYTES ((size_t)8 << 20)

int dpsgd_per_example_norms_multi_noalloc(const dpsgd_layer* layers, int32_t n_layers,
                                          int32_t mode, float* norms_sq, int32_t accumulate,
                                          void* stream);

/* ---------------------------------------------------------------------------
 * Clip factors.  Paper: Section 2.2, g_bar_i = g_i * min(1, C/||g_i||_2).
 *
 *   n_i = sqrt(norms_sq[i]);  factors[i] = n_i > C ? C / n_i : 1;
 *   mask[i] = n_i > C          (1 = clipped; a tie n_i == C is not clipped)
 * computed in float32. C must be > 0 (C = +inf disables clipping).
 * factors (float32 [B]) and mask (uint8 [B]) are device pointers; either may be NULL.
 * ------------------------------------------------------------------------- */
int dpsgd_clip_factors(const float* norms_sq, int64_t B, float C, float* factors,
                       uint8_t* mask, void* stream);

/* ---------------------------------------------------------------------------
 * Clipped sum.  Paper: Section 2.2 aggregation sum_i g_bar_i; GPU-side
 * algorithm, average step (the 1/B is left to dpsgd_add_noise's `scale`).
 *
 *   grad = (accumulate ? grad : 0) + sum_i c_i G_i^T A_i      (float32 [d_out][d_in])
 *
 * with c_i from dpsgd_clip_factors(norms_sq, B, C). factors_out / mask_out
 * (device, optional) receive c and the clip mask. The _multi form does the
 * same for n_layers layers (one grad buffer each, all with the same B) in one
 * grouped launch. workspace: at least dpsgd_clip_workspace_bytes(...) bytes,
 * 16-byte aligned (DPSGD_ERR_INVALID_ARG otherwise).
 * grad must be 16-byte aligned and must not alias any input.
 * ------------------------------------------------------------------------- */
size_t dpsgd_clip_workspace_bytes(const dpsgd_layer* layers, int32_t n_layers);

int dpsgd_clip_accumulate(const dpsgd_layer* layer, const float* norms_sq, float C,
                          float* grad, int32_t accumulate, float* factors_out,
                          uint8_t* mask_out, void* workspace, size_t workspace_bytes,
                          void* stream);

int dpsgd_clip_accumulate_multi(const dpsgd_layer* layers, int32_t n_layers,
                                const float* norms_sq, float C, float* const* grads,
                                int32_t accumulate, float* factors_out, uint8_t* mask_out,
                                void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Norms, factors and clipped sum in one call.  Paper: Section 2.2 (the
 * per-example norm over all layers, the clip factor and the sum of the
 * clipped gradients); GPU-side algorithm, clip and average steps.
 *
 *   norms_sq[i] = sum_l ||G_i^T A_i||_F^2            (float32 [B], overwritten)
 *   c_i, mask_i as in dpsgd_clip_factors(norms_sq, B, C)
 *   grads[l]    = (accumulate ? grads[l] : 0) + sum_i c_i G_i^T A_i
 *
 * the same results as dpsgd_per_example_norms_multi(..., accumulate = 0)
 * followed by dpsgd_clip_accumulate_multi, within float32 rounding. A layer
 * whose narrow side min(d_in, d_out) is at most 16 (a low-rank adapter
 * matrix), whose wide side is a multiple of 4 elements (at most 2^30) and
 * whose per-example gradient (4 d_in d_out bytes) is at most a quarter of its
 * per-example input bytes (T (d_in + d_out) element bytes) is read once:
 * every G_i^T A_i is formed in float32 and stored in the workspace, its
 * squared norm is summed from the stored values and the clipped sum is
 * formed from them. Other layers
 * use the kernels of the separate calls. mode applies to the other layers;
 * DPSGD_NORM_GHOST also turns the stored form off. workspace: at least
 * dpsgd_clipped_sum_workspace_bytes(layers, n_layers, mode) bytes (device,
 * 16-byte aligned; DPSGD_ERR_INVALID_ARG otherwise).
 * factors_out / mask_out are optional. Errors as in the two separate calls;
 * norms_sq must not be NULL.
 * ------------------------------------------------------------------------- */
size_t dpsgd_clipped_sum_workspace_bytes(const dpsgd_layer* layers, int32_t n_layers,
                                         int32_t mode);

int dpsgd_clipped_sum_multi(const dpsgd_layer* layers, int32_t n_layers, int32_t mode, float C,
                            float* const* grads, int32_t accumulate, float* norms_sq,
                            float* factors_out, uint8_t* mask_out, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Noise.  Paper: Section 2.2, z_t ~ N(0, sigma^2 C^2 I) and
 * g_tilde = (1/|B_t|)(sum + z_t); GPU-side algorithm, noise step
 * (g_tilde = g_bar + Noise(s_noise,t; sigma C)/B).
 *
 *   grad[e] = scale * (grad[e] + sigma * C * z_e),   e in [0, d_out*d_in)
 *
 * in place, float32. z_e is a standard normal from Philox4x32-10 (Salmon et
 * al., SC'11) and Box-Muller (1958): key = (seed mod 2^32, seed >> 32);
 * block j = e/4 has counter (j mod 2^32, j >> 32, layer->tensor_id, step);
 * from its words (r0,r1,r2,r3): u = ((r>>8)+1) 2^-24 for r0, r2 and
 * v = (r>>8) 2^-24 for r1, r3; z_{4j+0,1} = sqrt(-2 ln u_a)(cos, sin)(2 pi v_a),
 * z_{4j+2,3} likewise from (u_b, v_b). sigma == 0 gives exactly scale*grad.
 * Reads only d_in, d_out and tensor_id of the layer descriptor.
 * sigma >= 0, C > 0 and finite, scale finite. The layers of one _multi call
 * must have distinct tensor_ids (DPSGD_ERR_INVALID_ARG otherwise): layers
 * with the same id would get the same normals. Independence across calls is
 * the caller's: every (seed, tensor_id, step) must be used for one release
 * only.
 * ------------------------------------------------------------------------- */
int dpsgd_add_noise(const dpsgd_layer* layer, float* grad, float sigma, float C,
                    uint64_t seed, uint32_t step, float scale, void* stream);

int dpsgd_add_noise_multi(const dpsgd_layer* layers, int32_t n_layers, float* const* grads,
                          float sigma, float C, uint64_t seed, uint32_t step, float scale,
                          void* stream);

/* ---------------------------------------------------------------------------
 * Noise + AdamW step.  Paper: GPU-side algorithm, its last two steps (the
 * noisy average g_tilde = g_bar + Noise(s; sigma C)/B, then OptStep on it);
 * the update is the appendix's one-step AdamW map.
 *
 *   g          = scale * (grad[e] + sigma * C * z_e)       (z_e exactly as dpsgd_add_noise)
 *   m[e]      <- beta1 * m[e] + (1 - beta1) * g
 *   v[e]      <- beta2 * v[e] + (1 - beta2) * g * g
 *   param[e]  <- param[e] - lr * ( (m[e] / (1 - beta1^t)) / (sqrt(v[e] / (1 - beta2^t)) + eps)
 *                                  + weight_decay * param[e] )
 *   noisy_out[e] = g                                       (only when noisy_out is not NULL)
 *
 * for e in [0, d_out*d_in), in float32 (the bias corrections are formed in
 * double on the host). grad is read only. param, exp_avg (m), exp_avg_sq (v),
 * grad and noisy_out are float32 [d_out][d_in] device buffers, 16-byte
 * aligned, pairwise non-overlapping. The _multi form takes one pointer per
 * layer in each array; noisy_outs may be NULL (no layer writes g) or hold
 * NULL entries. The layer descriptor is read as in dpsgd_add_noise.
 * Errors (DPSGD_ERR_INVALID_ARG): a NULL or misaligned required pointer, the
 * noise arguments as in dpsgd_add_noise (distinct tensor_ids included), lr < 0
 * or not finite, beta1 or beta2
 * outside [0, 1), eps <= 0 or not finite, weight_decay < 0 or not finite,
 * t == 0.
 * ------------------------------------------------------------------------- */
typedef struct dpsgd_adamw {
  float lr;            /* learning rate eta_t of this step        */
  float beta1;         /* first-moment decay, in [0, 1)           */
  float beta2;         /* second-moment decay, in [0, 1)          */
  float eps;           /* added to sqrt(v_hat), > 0               */
  float weight_decay;  /* decoupled decay lambda, >= 0            */
  uint32_t t;          /* optimizer step, >= 1 (bias corrections) */
} dpsgd_adamw;

int dpsgd_noise_adamw(const dpsgd_layer* layer, const float* grad, float* param, float* exp_avg,
                      float* exp_avg_sq, float* noisy_out, float sigma, float C, uint64_t seed,
                      uint32_t step, float scale, const dpsgd_adamw* opt, void* stream);

int dpsgd_noise_adamw_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* grads, float* const* params,
                            float* const* exp_avgs, float* const* exp_avg_sqs,
                            float* const* noisy_outs, float sigma, float C, uint64_t seed,
                            uint32_t step, float scale, const dpsgd_adamw* opt, void* stream);

/* ---------------------------------------------------------------------------
 * Token tables (embeddings): lookup, per-example norms, clipped sum.
 * Paper: Section 2.2, per-example gradient of the trainable parameters, for
 * the one layer of a language model that is not of the G^T A form.
 *
 *   out[i][t]     = scale * table[id_it]                        (lookup)
 *   g_i[v]        = scale * sum_{t: id_it = v} G[i][t]          (gradient of example i)
 *
 * table [n_rows][d], ids [B][T], out and G [B][T][d], all row-major and
 * contiguous. An id outside [0, n_rows) is an empty position (padding): a row
 * of zeros in out, no part of the gradient; its row of G is not read.
 * A launch has fewer than 2^32 threads; calls that would need more are refused
 * (DPSGD_ERR_INVALID_ARG) with nothing enqueued. Never refused for it: lookups;
 * norms with B ceil(d / 1024) < 2^22 and n_rows <= 2^30; sums with
 * B T <= 2^28 - 32, n_rows <= 2^28 and B T ceil(d / 64) <= 2^30.
 * ids is aligned to its element, table, out and G to 16 bytes.
 * ------------------------------------------------------------------------- */
typedef enum dpsgd_index_dtype {
  DPSGD_I32 = 0,   /* int32 ids */
  DPSGD_I64 = 1    /* int64 ids */
} dpsgd_index_dtype;

typedef struct dpsgd_embedding {
  const void* ids;      /* [B][T] token ids, index_dtype                     */
  int64_t B;            /* examples, >= 1                                    */
  int64_t T;            /* positions per example, >= 1; B T <= 2^30          */
  int64_t n_rows;       /* rows of the table (vocabulary), 1 .. 2^31 - 1     */
  int64_t d;            /* width of a row, 1 .. 2^20                         */
  int32_t index_dtype;  /* dpsgd_index_dtype                                 */
  float scale;          /* finite                                            */
} dpsgd_embedding;

/* Products are formed in float32 and rounded once to out_dtype. table and out
 * are float32 or bf16 each on its own, and do not overlap. */
int dpsgd_embedding_lookup(const dpsgd_embedding* emb, const void* table, int32_t table_dtype,
                           void* out, int32_t out_dtype, void* stream);

/* Scratch of the two calls below (device, 16-byte aligned); 0 for an invalid
 * descriptor. Reads everything but ids of the descriptor. */
size_t dpsgd_embedding_workspace_bytes(const dpsgd_embedding* emb);

/* norms_sq[i] = (accumulate ? norms_sq[i] : 0) + ||g_i||_F^2 (float32 [B]):
 * with accumulate, the table joins the norm over the linear layers. dtype is
 * G's. Every group of equal tokens of an example is summed in float32 before
 * its squared norm is taken, and scale^2 multiplies the sum of squares. */
int dpsgd_embedding_norms(const dpsgd_embedding* emb, const void* G, int32_t dtype,
                          float* norms_sq, int32_t accumulate, void* workspace,
                          size_t workspace_bytes, void* stream);

/* grad = (accumulate ? grad : 0) + sum_i c_i g_i (float32 [n_rows][d], 16-byte
 * aligned), c_i, factors_out and mask_out as in dpsgd_clip_accumulate. norms_sq
 * NULL: every c_i is 1 (C is not looked at, factors_out and mask_out must be
 * NULL). norms_sq, grad, factors_out and mask_out do not overlap
 * (DPSGD_ERR_INVALID_ARG). Rows of examples with c_i = 0 are not read. Without accumulate every row
 * of grad is written, rows without a token with zeros. Sums are in float32,
 * in an order that the ids alone decide. */
int dpsgd_embedding_clip_accumulate(const dpsgd_embedding* emb, const void* G, int32_t dtype,
                                    const float* norms_sq, float C, float* grad,
                                    int32_t accumulate, float* factors_out, uint8_t* mask_out,
                                    void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Group norm with an activation, channels last.
 * Paper: Section 2.2 (a model trained by per-example gradients normalises
 * within an example).
 *
 *   x, y [B][S][C] (S positions: H W of an image, T of a sequence), groups of
 *   C / groups neighbouring channels; per example and group, over its
 *   S C / groups values:  mu = mean, rstd = 1 / sqrt(var + eps) (biased var)
 *   xh = (x - mu) rstd;  z = gamma xh + beta;  y = act(z)
 *
 * gamma and beta are float32 [C] (NULL: 1 and 0). Statistics and arithmetic
 * are float32; y is rounded once to dtype. x, y, dy, dx are contiguous and
 * 16-byte aligned.
 * A launch has fewer than 2^32 threads: 64 or more an example, up to four a
 * vector of channels of a row (4, 2 or 1 channels, the most that divides C), and
 * 256 a group where all rows of a group are no single tile. Calls that would
 * need more are refused (DPSGD_ERR_INVALID_ARG) with nothing enqueued.
 * ------------------------------------------------------------------------- */
typedef enum dpsgd_activation {
  DPSGD_ACT_NONE = 0,
  DPSGD_ACT_RELU = 1,   /* max(z, 0)                                                  */
  DPSGD_ACT_SILU = 2,   /* z / (1 + exp(-z))                                          */
  DPSGD_ACT_GELU = 3    /* 0.5 z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3)))            */
} dpsgd_activation;

typedef struct dpsgd_group_norm {
  int64_t B;            /* examples, >= 1                                    */
  int64_t S;            /* positions, >= 1; B S < 2^31                       */
  int64_t C;            /* channels, 1 .. 2^20, a multiple of groups         */
  int64_t groups;       /* >= 1                                              */
  const float* gamma;   /* [C], device; may be NULL                          */
  const float* beta;    /* [C], device; may be NULL                          */
  int32_t dtype;        /* dpsgd_dtype of x, y, dy, dx                       */
  int32_t act;          /* dpsgd_activation                                  */
  float eps;            /* > 0, finite                                       */
} dpsgd_group_norm;

/* Scratch of the two calls below (device, 16-byte aligned); 0 for an invalid
 * descriptor. Does not read the pointers of the descriptor. */
size_t dpsgd_group_norm_workspace_bytes(const dpsgd_group_norm* gn);

/* mean and rstd (float32 [B][groups]) are kept for the backward call; NULL
 * where there is none. y may be x. */
int dpsgd_group_norm_forward(const dpsgd_group_norm* gn, const void* x, void* y, float* mean,
                             float* rstd, void* workspace, size_t workspace_bytes, void* stream);

/* dx, and the per-example gradients of the affine parameters (float32 [B][C]):
 *   dz = dy act'(z);  dbeta[i] = sum_s dz;  dgamma[i] = sum_s dz xh
 *   dx = rstd (gamma dz - mean(gamma dz) - xh mean(gamma dz xh))
 * (means over the group; act'(0) = 0 for RELU). dgamma and dbeta are linear
 * layers' gradients with T = 1, d_in = 1, A = 1: a dpsgd_layer {A = ones [B],
 * G = dgamma} takes them through the norm, clip, noise and step calls. dx may
 * be dy, and may not be x. */
int dpsgd_group_norm_backward(const dpsgd_group_norm* gn, const void* x, const void* dy,
                              const float* mean, const float* rstd, void* dx, float* dgamma,
                              float* dbeta, void* workspace, size_t workspace_bytes,
                              void* stream);

/* ---------------------------------------------------------------------------
 * One norm over many tensors, and clipping to it.
 * Paper: Section 2.2, g min(1, C/||g||), with the whole of n_layers gradients
 * as one vector (one user's or one micro-batch's update; the released noisy
 * gradient before the optimizer step).
 *
 *   norm = sqrt(sum_l ||g_l||_F^2);  c = norm > max_norm ? max_norm / norm : 1
 *   outs[l] = c * grads[l]
 *
 * grads and outs: one float32 buffer of d_out d_in entries a layer, 16-byte
 * aligned; outs[l] may be grads[l] (in place), and overlaps nothing else. Only
 * d_in and d_out of a descriptor are read. Squares are summed in float64 and
 * the norm is rounded once to float32, infinite above its range; c is formed
 * from the norm before it is rounded. max_norm > 0 (+inf: c = 1, also for an
 * infinite norm). An infinite entry gives c = 0 under a finite max_norm (the
 * entry becomes NaN, finite ones 0), a NaN norm c = NaN. norm_out and
 * factor_out: float32 [1], device, either may be NULL in
 * dpsgd_global_clip_multi.
 * A launch has fewer than 2^32 threads: clipping takes up to 2^37 - 2^19 entries in
 * any 48 tensors in a row, and calls that would need more threads are refused
 * (DPSGD_ERR_INVALID_ARG) with nothing enqueued.
 * ------------------------------------------------------------------------- */
size_t dpsgd_global_norm_workspace_bytes(const dpsgd_layer* layers, int32_t n_layers);

int dpsgd_global_norm_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* grads, float* norm_out, void* workspace,
                            size_t workspace_bytes, void* stream);

int dpsgd_global_clip_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* grads, float* const* outs, float max_norm,
                            float* norm_out, float* factor_out, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Log probabilities of tokens, and the loss.
 * Paper: Section 2.2 (the per-example loss whose gradient is clipped), for a
 * language model or a classifier.
 *
 * logits: B T rows of V entries, float32 or bf16; row r begins at entry
 * r * stride, stride >= V (entries between V and stride are not read, nor
 * written in a gradient). Per row, in float32:
 *
 *   z = scale * logits;  m = max z;  S = sum_v exp(z_v - m)
 *   lse = m + ln S;  p_v = exp(z_v - m) / S;  logprob = (z_target - m) - ln S
 *   entropy = ln S - sum_v p_v (z_v - m)
 *
 *  - targets [B][T]; one outside [0, V) is an empty position (padding): its row
 *    is not read; logprob, lse and entropy are 0, it has no alternatives, and
 *    its gradient is a row of zeros. targets NULL: no position is empty, and
 *    there are no log probabilities of targets.
 *  - z_v = -inf (a masked token) has p_v = 0. A row whose every z is -inf has no
 *    distribution: lse and logprob are -inf, entropy 0, no alternatives, and the
 *    gradient is 0. A z of +inf or NaN makes the row's outputs and gradient NaN,
 *    without alternatives.
 * ------------------------------------------------------------------------- */
#define DPSGD_MOST_ALTERNATIVES 64

typedef struct dpsgd_logits {
  const void* targets;  /* [B][T] token ids, index_dtype; may be NULL        */
  int64_t B;            /* examples, >= 1                                    */
  int64_t T;            /* positions per example, >= 1; B T <= 2^30          */
  int64_t V;            /* tokens (classes), 1 .. 2^24                       */
  int64_t stride;       /* entries from a row to the next, V .. 2^31;
                           B T stride <= 2^40                                */
  int32_t index_dtype;  /* dpsgd_index_dtype                                 */
  int32_t dtype;        /* dpsgd_dtype of logits and their gradient          */
  float scale;          /* > 0, finite (1 / temperature)                     */
} dpsgd_logits;

/* Scratch of dpsgd_token_logprobs with k alternatives and of dpsgd_token_loss
 * (k = 0) (device, 16-byte aligned); 0 for an invalid descriptor or k. Does not
 * read targets. */
size_t dpsgd_token_workspace_bytes(const dpsgd_logits* desc, int32_t k);

/* logprobs, lse, entropy: float32 [B][T]. top_ids (int64) and top_logprobs
 * (float32) [B][T][k]: the k largest logits of a row and their log
 * probabilities, largest first, of equal logits the lower token first; where a
 * row has fewer than k logits above -inf, id -1 and -inf follow (NaN instead of
 * -inf where the row is NaN). 0 <= k <= DPSGD_MOST_ALTERNATIVES; with k = 0
 * top_ids and top_logprobs must be NULL. Any output may be NULL, not all; with
 * targets NULL logprobs must be. logits is aligned to its element. */
int dpsgd_token_logprobs(const dpsgd_logits* desc, const void* logits, float* logprobs, float* lse,
                         float* entropy, int32_t k, int64_t* top_ids, float* top_logprobs,
                         void* workspace, size_t workspace_bytes, void* stream);

/* The gradient of sum grad_logprobs logprob + grad_lse lse + grad_entropy entropy
 * (each float32 [B][T]; NULL: 0, not all of them) by the logits, rounded once to
 * dtype:
 *   dlogits_v = scale (p_v (grad_lse - grad_logprobs - grad_entropy (ln p_v + entropy))
 *                      + grad_logprobs [v = target])
 * lse and entropy are dpsgd_token_logprobs' (entropy is read only with
 * grad_entropy). p_v is exp(z_v - lse) where lse is within 32 of 0 (1024 in bf16),
 * so that its rounding is lost in dtype's; beyond, m and S are formed again from
 * the logits. A row whose three factors are 0 gets zeros, whatever its
 * logits. Row r of dlogits begins at entry r * dlogits_stride (V .. 2^31).
 * dlogits may be logits (with the same stride), and overlaps nothing else. */
int dpsgd_token_logprobs_backward(const dpsgd_logits* desc, const void* logits, const float* lse,
                                  const float* entropy, const float* grad_logprobs,
                                  const float* grad_lse, const float* grad_entropy, void* dlogits,
                                  int64_t dlogits_stride, void* stream);

/* Per-example losses and the gradient of their sum, the logits read once where a
 * row fits a workgroup's registers (V up to 131072 in bf16, 65536 in float32):
 *   losses[i] = -sum_t w_it logprob_it                     (float32 [B], or NULL)
 *   dlogits   = scale w_it (p_v - [v = target])            as above
 * weights float32 [B][T]; NULL: all 1. A position of weight 0 adds nothing and
 * gets zeros, whatever its logits. logprobs (float32 [B][T]) may be NULL.
 * targets must not be NULL. */
int dpsgd_token_loss(const dpsgd_logits* desc, const void* logits, const float* weights,
                     float* losses, float* logprobs, void* dlogits, int64_t dlogits_stride,
                     void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * The residual sum between two blocks, with the norms on both sides of it.
 * Paper: Section 2.2, per-example gradients of the trainable parameters.
 *
 *   u = post ? norm(block) post_gamma + post_beta : block
 *   r = residual_scale x + gate u            (rounded to dtype)
 *   y = norm(r) gamma + beta                 (of r as it is stored)
 *   norm(v) = (v - mean) rstd, rstd = 1 / sqrt(var + eps)      (LAYER)
 *           = v rstd, rstd = 1 / sqrt(mean(v^2) + eps)         (RMS)
 *
 * over rows of C channels; x, block, r, y [B][S][C], contiguous. block NULL: r =
 * residual_scale x, with no gate and no post. Arithmetic and statistics are
 * float32; r and y are rounded once each. Every tensor, the affine parameters and
 * their gradients among them, is 16-byte aligned.
 * ------------------------------------------------------------------------- */
typedef enum dpsgd_row_norm {
  DPSGD_ROW_NORM_LAYER = 0,
  DPSGD_ROW_NORM_RMS = 1
} dpsgd_row_norm;

typedef struct dpsgd_residual_norm {
  int64_t B;                 /* examples, >= 1                                    */
  int64_t S;                 /* positions per example, >= 1; B S < 2^31           */
  int64_t C;                 /* channels, 1 .. 16384                              */
  const float* gamma;        /* [C], device; NULL: 1                              */
  const float* beta;         /* [C], device; NULL: 0                              */
  const float* post_gamma;   /* the same for the block's norm; NULL without post  */
  const float* post_beta;
  const float* gate;         /* NULL: 1; [C], or [B][C] with gate_per_example     */
  int32_t gate_per_example;
  int32_t post;              /* the block's output is normed before it is added   */
  int32_t kind;              /* dpsgd_row_norm of both norms                      */
  int32_t dtype;             /* dpsgd_dtype of x, block, r, y and their gradients */
  float residual_scale;      /* finite                                            */
  float eps;                 /* > 0, finite                                       */
} dpsgd_residual_norm;

/* stats (float32 [B][S][4]: mean, rstd of r, mean, rstd of the block's output; 0
 * where there is none) is kept for the backward call; NULL
 * where there is none. r may be x and y may be block; r may be NULL (not
 * written; y is formed from the same rounded values). Outputs overlap nothing
 * else. */
int dpsgd_residual_norm_forward(const dpsgd_residual_norm* desc, const void* x, const void* block,
                                void* r, void* y, float* stats, void* stream);

/* Scratch of the call below (device, 16-byte aligned); 0 for an invalid
 * descriptor. Does not read the pointers of the descriptor. */
size_t dpsgd_residual_norm_workspace_bytes(const dpsgd_residual_norm* desc);

/* From dy and dr (the gradient that reaches r past the norm; NULL: 0), with
 * D(g, vh) the norm's backward, rstd (g - mean(g) - vh mean(g vh)) (RMS: without
 * mean(g)):
 *   dR = dr + D(dy gamma, rh);  dx = residual_scale dR;  dU = gate dR
 *   dblock = post ? D(dU post_gamma, bh) : dU
 * and the per-example gradients (float32 [B][C], each may be NULL: not formed)
 *   dgamma_i = sum_s dy rh;  dbeta_i = sum_s dy;  dgate_i = sum_s dR u
 *   dpost_gamma_i = sum_s dU bh;  dpost_beta_i = sum_s dU
 * which the norm, clip, noise and step calls take as layers with T = 1, d_in = 1,
 * A = 1. block and dblock are NULL together; block is not read without post and
 * dgate. r is the forward call's (x for a block NULL with residual_scale 1).
 * dx may be dr or NULL, dblock may be dy; they overlap nothing else. A launch has
 * fewer than 2^32 threads, 64 to 1024 for each example at least; calls that would
 * need more are refused (DPSGD_ERR_INVALID_ARG; never with B < 2^22) with nothing
 * enqueued. */
int dpsgd_residual_norm_backward(const dpsgd_residual_norm* desc, const void* block, const void* r,
                                 const void* dy, const void* dr, const float* stats, void* dx,
                                 void* dblock, float* dgamma, float* dbeta, float* dgate,
                                 float* dpost_gamma, float* dpost_beta, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Noise + AdamW step with moments in 8 bits.
 * Paper: GPU-side algorithm, its last two steps, as dpsgd_noise_adamw.
 *
 * The moments of a tensor of n entries are n codes each, and a pair of exponents
 * (k_m, k_v, uint8, biased by 127) for every 256 entries in a row:
 *   m: bit 7 the sign, bits 6..3 an exponent E, bits 2..0 a fraction F
 *      |m| = (1 + F/8) 2^(E - 15 + k_m - 127),  E = 0: F/8 2^(-14 + k_m - 127)
 *   v: bits 7..3 E, bits 2..0 F
 *      v = (1 + F/8) 2^(E - 31 + k_v - 127),    E = 0: F/8 2^(-30 + k_v - 127)
 * All zeros stand for moments of 0. A block's exponent is that of its largest
 * magnitude rounded up to 3 bits of fraction, at least 32 (m) or 48 (v); the
 * exponent 255 stands for a block with a magnitude that is not finite (or is
 * above 1.875 2^127), which reads back as NaN.
 *
 * One step, every operation rounded to float32 by itself (no fused multiply-add;
 * the constants are formed in double on the host and rounded):
 *   g = scale * (grad + sigma C z)                (z, and its sum, as dpsgd_noise_adamw)
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) (g g)
 *   param = param (1 - lr weight_decay)
 *           - (m / (sqrt(v) (1 / sqrt(1 - beta2^t)) + eps)) (lr / (1 - beta1^t))
 * with m and v in float32, which are then rounded to codes:
 *  - DPSGD_ROUND_NEAREST: to nearest, ties to even.
 *  - DPSGD_ROUND_STOCHASTIC: up with the probability of the distance from the
 *    value below, in steps of 2^-16 (the mean of many steps is kept, which nearest
 *    rounding loses for changes of less than half a code, as most of v's are).
 *    Entry e takes word e mod 4 of the Philox4x32-10 block j = e / 4 with counter
 *    (j mod 2^32, j >> 32, tensor_id, t) and the complement of round_seed as its
 *    key: bits 0..15 for m, 16..31 for v.
 * A v above 0 is never rounded to 0.
 * ------------------------------------------------------------------------- */
#define DPSGD_STATE_BLOCK 256

typedef enum dpsgd_rounding {
  DPSGD_ROUND_NEAREST = 0,
  DPSGD_ROUND_STOCHASTIC = 1
} dpsgd_rounding;

/* Arrays and arguments as in dpsgd_noise_adamw_multi; exp_avgs and exp_avg_sqs
 * hold codes (uint8 [d_out d_in]), exponents uint8 [ceil(d_out d_in / 256)][2],
 * all 16-byte aligned and pairwise non-overlapping. round_seed is read only with
 * DPSGD_ROUND_STOCHASTIC. A launch has fewer than 2^32 threads: any 48 tensors in a
 * row have up to 2^35 entries together (less 2^18 for their ends), and calls that
 * would need more are refused, with nothing enqueued. */
int dpsgd_noise_adamw8_multi(const dpsgd_layer* layers, int32_t n_layers,
                             const float* const* grads, float* const* params,
                             uint8_t* const* exp_avgs, uint8_t* const* exp_avg_sqs,
                             uint8_t* const* exponents, float* const* noisy_outs, float sigma,
                             float C, uint64_t seed, uint32_t step, float scale,
                             const dpsgd_adamw* opt, int32_t rounding, uint64_t round_seed,
                             void* stream);

/* float32 moments (v >= 0) to codes and exponents, to nearest, and codes to
 * moments, float32 or bf16 (both exact). A NaN, infinite or (v) negative
 * moment makes its block NaN. */
int dpsgd_adamw8_pack_multi(const dpsgd_layer* layers, int32_t n_layers,
                            const float* const* exp_avgs_in, const float* const* exp_avg_sqs_in,
                            uint8_t* const* exp_avgs, uint8_t* const* exp_avg_sqs,
                            uint8_t* const* exponents, void* stream);
int dpsgd_adamw8_unpack_multi(const dpsgd_layer* layers, int32_t n_layers,
                              const uint8_t* const* exp_avgs, const uint8_t* const* exp_avg_sqs,
                              const uint8_t* const* exponents, void* const* exp_avgs_out,
                              void* const* exp_avg_sqs_out, int32_t out_dtype, void* stream);

/* ---------------------------------------------------------------------------
 * Inspection hooks for tests (same stream as dpsgd_add_noise).
 *   dpsgd_philox_u32: out[4*b + w] = word w of block (first_block + b), b < n_blocks.
 *   dpsgd_gaussian:   out[e] = z_e of the stream above for e < n.
 * out is a device pointer.
 * ------------------------------------------------------------------------- */
int dpsgd_philox_u32(uint32_t* out, int64_t first_block, int64_t n_blocks, uint64_t seed,
                     uint32_t tensor_id, uint32_t step, void* stream);
int dpsgd_gaussian(float* out, int64_t n, uint64_t seed, uint32_t tensor_id, uint32_t step,
                   void* stream);

/* Static text for a dpsgd_status value. */
const char* dpsgd_status_string(int status);

/* Library version, for the binding's load check. */
int dpsgd_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DPSGD_H_ */
