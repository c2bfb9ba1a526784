// The norm over many float32 tensors, and the tensors scaled to at most a given
// norm:
//
//   n = sqrt(sum_l ||g_l||^2),  c = n > max_norm ? max_norm / n : 1,  out_l = c g_l
//
// Bound by memory traffic: the tensors are read once for the norm and, since
// the factor needs all of it, once more to be scaled. Squares are summed in
// float64: the conversion and the fused multiply-add are far below the memory
// time, no square overflows or vanishes, and the norm is rounded once.
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

constexpr int kBlock = 4096;        // entries that a workgroup takes at a time
constexpr int kNormWgs = 1024;      // most workgroups (partial sums) of a launch

struct Tensor {
  const float* in;
  float* out;
  int64_t numel;
  int64_t begin;   // first block of this tensor in the launch
};

struct ClipArgs {
  Tensor t[kMaxLayersPerLaunch];
  int64_t blocks;
  double* partials;     // of this launch
  const float* factor;
  int32_t n;
};

__device__ __forceinline__ const Tensor& tensor_of(const ClipArgs& a, int64_t block) {
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].begin <= block) lo = mid; else hi = mid - 1;
  }
  return a.t[lo];
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

__global__ __launch_bounds__(kThreads) void sum_squares_kernel(ClipArgs a) {
  __shared__ double red[kThreads / 64];
  double s = 0.0;
  for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) {
    const Tensor& t = tensor_of(a, b);
    const int64_t e0 = (b - t.begin) * kBlock;
    for (int k = 0; k < kBlock / (4 * kThreads); ++k) {
      const int64_t e = e0 + (k * kThreads + (int)threadIdx.x) * 4;
      if (e + 4 <= t.numel) {
        float x[4];
        load_vec<4>(t.in + e, x);
#pragma unroll
        for (int c = 0; c < 4; ++c) s = fma((double)x[c], (double)x[c], s);
      } else {
        for (int64_t q = e; q < t.numel; ++q) s = fma((double)t.in[q], (double)t.in[q], s);
      }
    }
  }
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.partials[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// The norm and the factor from all partial sums.
__global__ __launch_bounds__(kThreads) void norm_finish_kernel(const double* partials, int64_t n,
                                                               float max_norm, float* norm_out,
                                                               float* factor, float* factor_out) {
  __shared__ double red[kThreads / 64];
  double s = 0.0;
  for (int64_t k = threadIdx.x; k < n; k += kThreads) s += partials[k];
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  const double norm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  if (norm_out) *norm_out = (float)norm;
  const float c = norm > (double)max_norm ? (float)((double)max_norm / norm)
                                          : (norm == norm ? 1.0f : (float)norm);
  if (factor) *factor = c;
  if (factor_out) *factor_out = c;
}

__global__ __launch_bounds__(kThreads) void scale_kernel(ClipArgs a) {
  const float c = *a.factor;
  const int64_t b = blockIdx.x;
  const Tensor& t = tensor_of(a, b);
  const int64_t e0 = (b - t.begin) * kBlock;
  for (int k = 0; k < kBlock / (4 * kThreads); ++k) {
    const int64_t e = e0 + (k * kThreads + (int)threadIdx.x) * 4;
    if (e + 4 <= t.numel) {
      float x[4];
      load_vec<4>(t.in + e, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= c;
      store_vec<4>(t.out + e, x);
    } else {
      for (int64_t q = e; q < t.numel; ++q) t.out[q] = t.in[q] * c;
    }
  }
}

// The launch over the tensors [base, base + n).
ClipArgs args_of(const dpsgd_layer* layers, int32_t n, const float* const* in, float* const* out) {
  ClipArgs a{};
  a.n = n;
  for (int32_t l = 0; l < n; ++l) {
    const int64_t numel = layers[l].d_in * layers[l].d_out;
    a.t[l] = Tensor{in ? in[l] : nullptr, out ? out[l] : nullptr, numel, a.blocks};
    a.blocks += ceil_div(numel, kBlock);
  }
  return a;
}

int64_t norm_wgs(const ClipArgs& a) { return a.blocks < kNormWgs ? a.blocks : kNormWgs; }

}  // namespace

// Workspace: the factor, then one float64 partial sum per workgroup.
size_t global_norm_workspace_bytes(const dpsgd_layer* layers, int32_t n) {
  int64_t partials = 0;
  for (int32_t base = 0; base < n; base += kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    partials += norm_wgs(args_of(layers + base, m, nullptr, nullptr));
  }
  return 256 + (size_t)partials * sizeof(double);
}

int launch_global_clip(const dpsgd_layer* layers, int32_t n, const float* const* grads,
                       float* const* outs, float max_norm, float* norm_out, float* factor_out,
                       void* workspace, hipStream_t stream) {
  float* factor = static_cast<float*>(workspace);
  double* partials = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
  int64_t at = 0;
  for (int32_t base = 0; base < n; base += kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    ClipArgs a = args_of(layers + base, m, grads + base, nullptr);
    if (a.blocks > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
    a.partials = partials + at;
    hipLaunchKernelGGL(sum_squares_kernel, dim3((uint32_t)norm_wgs(a)), dim3(kThreads), 0, stream, a);
    at += norm_wgs(a);
  }
  hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kThreads), 0, stream, partials, at, max_norm,
                     norm_out, factor, factor_out);
  if (!outs) return check_launch();
  for (int32_t base = 0; base < n; base += kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    ClipArgs a = args_of(layers + base, m, grads + base, outs + base);
    a.factor = factor;
    hipLaunchKernelGGL(scale_kernel, dim3((uint32_t)a.blocks), dim3(kThreads), 0, stream, a);
  }
  return check_launch();
}

}  // namespace dpsgd
