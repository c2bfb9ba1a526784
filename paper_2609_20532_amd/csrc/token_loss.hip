// Log probabilities of tokens, entropy, the most likely tokens, and the loss with its
// gradient, over rows of V logits:
//
//   z = scale x;  m = max z;  d = z - m;  S = sum e^d;  E = sum e^d d
//   lse = m + ln S;  logp = d_target - ln S;  entropy = ln S - E / S
//   dx_v = scale (p_v (g_lse - g_logp - g_H (ln p_v + H)) + g_logp [v = target])
//
// Bound by memory traffic: each logit is read once, and written once in a gradient.
#include <math.h>

#include "vec.h"

// z - m is formed from the rounded product z: contracted, it could be above 0 by a
// rounding of z, which is any number for logits far from 0.
#pragma clang fp contract(off)

namespace dpsgd {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int64_t kMostWgs = 1 << 20;

struct TokenArgs {
  const void* logits;
  const void* targets;        // may be null
  void* dlogits;
  const float* weights;       // null: 1
  const float* lse;           // backward
  const float* entropy;
  const float* g_logp;
  const float* g_lse;
  const float* g_entropy;
  float* logp_out;            // the outputs may be null
  float* lse_out;
  float* entropy_out;
  int64_t* top_ids;
  float* top_logprobs;
  int64_t rows, stride, grad_stride;
  int32_t V, k, wide_ids;
  float scale;
};

// e^d for d <= 0: exactly 0 for -inf.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// The target of a row, -1 for an empty position; *empty: there is none.
__device__ __forceinline__ int32_t target_of(const TokenArgs& a, int64_t row, bool* empty) {
  *empty = false;
  if (!a.targets) return -1;
  const int64_t t = a.wide_ids ? static_cast<const int64_t*>(a.targets)[row]
                               : (int64_t)static_cast<const int32_t*>(a.targets)[row];
  *empty = t < 0 || t >= a.V;
  return *empty ? -1 : (int32_t)t;
}

template <class T>
__device__ __forceinline__ float entry(const T* x, int32_t v) {
  float f[1];
  load_vec<1>(x + v, f);
  return f[0];
}

template <class T>
__device__ __forceinline__ void put(T* x, int32_t v, float value) {
  const float f[1] = {value};
  store_vec<1>(x + v, f);
}

// An order of logits (the larger first, of equal ones the lower token) as whole
// numbers; 0 is below every logit.
__device__ __forceinline__ uint64_t order_of(float x, int32_t v) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // -0 as 0
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (uint32_t)~v;
}

__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  const float r = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  __syncthreads();
  return r;
}

__device__ __forceinline__ uint64_t block_max_u64(uint64_t v, uint64_t* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)v, off, 64);
    v = o > v ? o : v;
  }
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t r = red[0];
  for (int w = 1; w < 4; ++w) r = red[w] > r ? red[w] : r;
  __syncthreads();
  return r;
}

// A row's statistics.
struct RowStats {
  float m, sum, log_sum, entropy;
  bool nan, none;   // NaN or +inf; all -inf
};

template <class T>
__device__ __forceinline__ RowStats stats_of(const TokenArgs& a, const T* x, float* red) {
  float m = -INFINITY;
  for (int32_t v = threadIdx.x; v < a.V; v += kThreads) m = fmaxf(m, a.scale * entry(x, v));
  m = block_max(m, red);
  const float m0 = m == -INFINITY ? 0.0f : m;
  float s = 0.0f, e = 0.0f;
  for (int32_t v = threadIdx.x; v < a.V; v += kThreads) {
    const float d = a.scale * entry(x, v) - m0, p = exp_of(d);
    s += p;
    e += p == 0.0f ? 0.0f : p * d;
  }
  s = block_sum(s, red);
  e = block_sum(e, red);
  RowStats st;
  st.nan = !(s == s) || m == INFINITY;
  st.none = !st.nan && m == -INFINITY;
  st.m = m;
  st.sum = s;
  st.log_sum = logf(s);
  st.entropy = st.nan ? NAN : (st.none ? 0.0f : st.log_sum - e / s);
  return st;
}

__device__ __forceinline__ float logp_of(const RowStats& st, float z) {
  return st.nan ? NAN : (st.none ? -INFINITY : (z - st.m) - st.log_sum);
}

template <class T>
__global__ __launch_bounds__(kThreads) void token_row_kernel(TokenArgs a) {
  __shared__ float red[4];
  __shared__ uint64_t red64[4];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    RowStats st{};
    if (!empty) st = stats_of(a, x, red);
    if (threadIdx.x == 0) {
      if (a.logp_out) a.logp_out[row] = empty ? 0.0f : logp_of(st, a.scale * entry(x, target));
      if (a.lse_out) a.lse_out[row] = empty ? 0.0f : (st.nan ? NAN : (st.none ? -INFINITY : st.m + st.log_sum));
      if (a.entropy_out) a.entropy_out[row] = empty ? 0.0f : st.entropy;
    }
    uint64_t last = ~(uint64_t)0;
    for (int32_t i = 0; i < a.k; ++i) {
      uint64_t best = 0;
      if (!empty && !st.nan && !st.none) {
        for (int32_t v = threadIdx.x; v < a.V; v += kThreads) {
          const float f = entry(x, v);
          const uint64_t o = order_of(f, v);
          if (f > -INFINITY && o < last && o > best) best = o;
        }
        best = block_max_u64(best, red64);
        last = best;
      }
      if (threadIdx.x == 0) {
        const int32_t v = best ? (int32_t)~(uint32_t)best : -1;
        if (a.top_ids) a.top_ids[row * a.k + i] = v;
        if (a.top_logprobs)
          a.top_logprobs[row * a.k + i] =
              best ? logp_of(st, a.scale * entry(x, v)) : (st.nan ? NAN : -INFINITY);
      }
    }
    if (a.dlogits) {
      __syncthreads();   // dlogits may be logits
      T* g = static_cast<T*>(a.dlogits) + row * a.grad_stride;
      const float w = empty ? 0.0f : (a.weights ? a.weights[row] : 1.0f);
      const float f = st.none ? 0.0f : a.scale * w, inv = 1.0f / st.sum;
      for (int32_t v = threadIdx.x; v < a.V; v += kThreads) {
        float out = 0.0f;
        if (w != 0.0f && st.nan) out = NAN;
        if (w != 0.0f && !st.nan && !st.none)
          out = f * (exp_of(a.scale * entry(x, v) - st.m) * inv - (v == target ? 1.0f : 0.0f));
        put(g, v, out);
      }
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void token_backward_kernel(TokenArgs a) {
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    T* g = static_cast<T*>(a.dlogits) + row * a.grad_stride;
    bool empty;
    const int32_t target = target_of(a, row, &empty);
    const float gp = empty || !a.g_logp ? 0.0f : a.g_logp[row];
    const float gl = empty || !a.g_lse ? 0.0f : a.g_lse[row];
    const float ge = empty || !a.g_entropy ? 0.0f : a.g_entropy[row];
    const bool zero = gp == 0.0f && gl == 0.0f && ge == 0.0f;
    const float lse = zero ? 0.0f : a.lse[row], H = ge != 0.0f ? a.entropy[row] : 0.0f;
    const bool none = lse == -INFINITY;
    for (int32_t v = threadIdx.x; v < a.V; v += kThreads) {
      float out = 0.0f;
      if (!zero && !none) {
        const float l = a.scale * entry(x, v) - lse, p = exp_of(l);
        float q = gl - gp;
        if (ge != 0.0f && p != 0.0f) q -= ge * (l + H);
        out = a.scale * (p * q + (v == target ? gp : 0.0f));
      }
      put(g, v, out);
    }
  }
}

// losses[i] = -sum_t w logp, one wave an example.
__global__ __launch_bounds__(kThreads) void token_losses_kernel(TokenArgs a, const float* logp,
                                                                float* losses, int64_t B, int64_t T) {
  const int lane = threadIdx.x & 63;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < B; i += (int64_t)gridDim.x * 4) {
    float s = 0.0f;
    for (int64_t t = lane; t < T; t += 64) {
      const int64_t row = i * T + t;
      bool empty;
      target_of(a, row, &empty);
      const float w = empty ? 0.0f : (a.weights ? a.weights[row] : 1.0f);
      if (w != 0.0f) s = fmaf(-w, logp[row], s);
    }
    s = wave_total(s);
    if (lane == 0) losses[i] = s;
  }
}

TokenArgs common_args(const dpsgd_logits& d, const void* logits) {
  TokenArgs a{};
  a.logits = logits;
  a.targets = d.targets;
  a.rows = d.B * d.T;
  a.stride = d.stride;
  a.V = (int32_t)d.V;
  a.wide_ids = d.index_dtype == DPSGD_I64;
  a.scale = d.scale;
  return a;
}

uint32_t grid_of(int64_t n) { return (uint32_t)(n < kMostWgs ? n : kMostWgs); }

int launch_rows(const TokenArgs& a, int32_t dtype, hipStream_t stream) {
  if (dtype == DPSGD_BF16)
    hipLaunchKernelGGL(token_row_kernel<uint16_t>, dim3(grid_of(a.rows)), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(token_row_kernel<float>, dim3(grid_of(a.rows)), dim3(kThreads), 0, stream, a);
  return check_launch();
}

}  // namespace

size_t token_workspace_bytes(const dpsgd_logits& d, int32_t k) {
  (void)k;
  return round_up((size_t)(d.B * d.T) * sizeof(float), 16);
}

int launch_token_logprobs(const dpsgd_logits& d, const void* logits, float* logprobs, float* lse,
                          float* entropy, int32_t k, int64_t* top_ids, float* top_logprobs,
                          void* workspace, hipStream_t stream) {
  (void)workspace;
  TokenArgs a = common_args(d, logits);
  a.logp_out = logprobs;
  a.lse_out = lse;
  a.entropy_out = entropy;
  a.k = k;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  return launch_rows(a, d.dtype, stream);
}

int launch_token_backward(const dpsgd_logits& d, const void* logits, const float* lse,
                          const float* entropy, const float* g_logp, const float* g_lse,
                          const float* g_entropy, void* dlogits, int64_t dlogits_stride,
                          hipStream_t stream) {
  TokenArgs a = common_args(d, logits);
  a.lse = lse;
  a.entropy = entropy;
  a.g_logp = g_logp;
  a.g_lse = g_lse;
  a.g_entropy = g_entropy;
  a.dlogits = dlogits;
  a.grad_stride = dlogits_stride;
  if (d.dtype == DPSGD_BF16)
    hipLaunchKernelGGL(token_backward_kernel<uint16_t>, dim3(grid_of(a.rows)), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(token_backward_kernel<float>, dim3(grid_of(a.rows)), dim3(kThreads), 0, stream, a);
  return check_launch();
}

int launch_token_loss(const dpsgd_logits& d, const void* logits, const float* weights,
                      float* losses, float* logprobs, void* dlogits, int64_t dlogits_stride,
                      void* workspace, hipStream_t stream) {
  TokenArgs a = common_args(d, logits);
  a.weights = weights;
  a.dlogits = dlogits;
  a.grad_stride = dlogits_stride;
  a.logp_out = logprobs ? logprobs : static_cast<float*>(workspace);
  const int st = launch_rows(a, d.dtype, stream);
  if (st != DPSGD_OK || !losses) return st;
  hipLaunchKernelGGL(token_losses_kernel, dim3(grid_of(ceil_div(d.B, 4))), dim3(kThreads), 0,
                     stream, a, a.logp_out, losses, d.B, d.T);
  return check_launch();
}

}  // namespace dpsgd
