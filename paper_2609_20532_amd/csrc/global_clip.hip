// The norm over many float32 tensors, and the tensors scaled to at most a given
// norm:
//
//   n = sqrt(sum_l ||g_l||^2),  c = n > max_norm ? max_norm / n : 1,  out_l = c g_l
//
// Bound by memory traffic: the tensors are read once for the norm and, since
// the factor needs all of it, once more to be scaled. Squares are summed in
// float64: the conversion and the fused multiply-add are far below the memory
// time, no square overflows or vanishes, and the norm is rounded once. Every
// workgroup of the second pass adds up the first one's partial sums itself: two
// launches. 48 tensors of 340 MB: 58 us (5.9 TB/s) and 110 us (680 MB, 6.2 TB/s);
// 24 tensors of 0.59 MB: 4.6 and 6.7 us.
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

constexpr int kBlock = 8192;        // entries that a workgroup takes at a time
constexpr int kNormWgs = 2048;      // most workgroups (partial sums) of a launch
// Outputs apart from the inputs that are this large together are written past
// the caches: they would displace, in the 256 MB last-level cache, what this call
// still has to read, and would mostly be gone again when they are used. Noise,
// clip and AdamW over 340 MB take 672 us so, 682 otherwise (the clip alone 168
// and 196); over 170 MB there is no difference, over 113 MB they take 227 and
// 223, and in place (where the lines are there already) 168 and 165 for 340 MB.
constexpr int64_t kPastCaches = INT64_C(192) << 20;
constexpr int kPerThread = kBlock / (4 * kThreads);

struct Tensor {
  const float* in;
  float* out;
  int64_t numel;
  int64_t begin;   // first block of this tensor in the launch
};

struct ClipArgs {
  Tensor t[kMaxLayersPerLaunch];
  int64_t blocks;
  double* partials;      // of this launch
  const double* all;     // scale: the partial sums of every launch, and their number
  int64_t n_all;
  float* norm_out;
  float* factor_out;
  float max_norm;
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

// Sum over the workgroup, in every thread.
__device__ __forceinline__ double block_sum_f64(double v) {
  __shared__ double red[kThreads / 64];
  v = wave_sum_f64(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kThreads) void sum_squares_kernel(ClipArgs a) {
  double s = 0.0;
  int64_t b = blockIdx.x;
  Tensor t = tensor_of(a, b);   // a workgroup's first block is there
  while (true) {
    const int64_t first = (b - t.begin) * kBlock, e0 = first + (int64_t)threadIdx.x * 4;
    float x[kPerThread][4];
    if (first + kBlock <= t.numel) {
#pragma unroll
      for (int k = 0; k < kPerThread; ++k) load_vec<4>(t.in + e0 + k * 4 * kThreads, x[k]);
    } else {
#pragma unroll
      for (int k = 0; k < kPerThread; ++k)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int64_t e = e0 + k * 4 * kThreads + c;
          x[k][c] = e < t.numel ? t.in[e] : 0.0f;
        }
    }
    b += gridDim.x;
    const bool more = b < a.blocks;
    if (more) t = tensor_of(a, b);   // while the loads are in flight
#pragma unroll
    for (int k = 0; k < kPerThread; ++k)
#pragma unroll
      for (int c = 0; c < 4; ++c) s = fma((double)x[k][c], (double)x[k][c], s);
    if (!more) break;
  }
  s = block_sum_f64(s);
  if (threadIdx.x == 0) a.partials[blockIdx.x] = s;
}

// The norm from the partial sums of every launch: each workgroup adds them for
// itself, in the same order.
__device__ __forceinline__ double norm_of(const ClipArgs& a) {
  double s = 0.0;
#pragma unroll 8
  for (int64_t k = threadIdx.x; k < a.n_all; k += kThreads) s += a.all[k];
  return sqrt(block_sum_f64(s));
}

__global__ __launch_bounds__(kThreads) void norm_kernel(ClipArgs a) {
  const double norm = norm_of(a);
  if (threadIdx.x == 0) *a.norm_out = (float)norm;
}

// PAST_CACHES: the outputs are not kept in the caches.
template <bool PAST_CACHES>
__global__ __launch_bounds__(kThreads) void scale_kernel(ClipArgs a) {
  // Last blocks first: they are the ones that the norm's pass has left in the
  // last-level cache (340 MB: 110 us, 118 in plain order).
  const int64_t b = a.blocks - 1 - blockIdx.x;
  const Tensor& t = tensor_of(a, b);
  const int64_t e0 = (b - t.begin) * kBlock + (int64_t)threadIdx.x * 4;
  const bool whole = e0 - (int64_t)threadIdx.x * 4 + kBlock <= t.numel;
  float x[kPerThread][4];
  if (whole) {
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) load_vec<4>(t.in + e0 + k * 4 * kThreads, x[k]);
  }
  const double norm = norm_of(a);
  const float c = norm > (double)a.max_norm ? (float)((double)a.max_norm / norm)
                                            : (norm == norm ? 1.0f : (float)norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (a.norm_out) *a.norm_out = (float)norm;
    if (a.factor_out) *a.factor_out = c;
  }
  if (whole) {
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[k][j] *= c;
      const f32x4_t y{x[k][0], x[k][1], x[k][2], x[k][3]};
      f32x4_t* to = reinterpret_cast<f32x4_t*>(t.out + e0 + k * 4 * kThreads);
      if constexpr (PAST_CACHES) __builtin_nontemporal_store(y, to);
      else *to = y;
    }
    return;
  }
  for (int k = 0; k < kPerThread; ++k)
    for (int j = 0; j < 4; ++j) {
      const int64_t e = e0 + k * 4 * kThreads + j;
      if (e < t.numel) t.out[e] = t.in[e] * c;
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

// Workgroups of the norm's pass: as few blocks each as kNormWgs allow, and the
// same number for nearly all.
int64_t norm_wgs(const ClipArgs& a) { return ceil_div(a.blocks, ceil_div(a.blocks, kNormWgs)); }

}  // namespace

// Workspace: one float64 partial sum per workgroup.
size_t global_norm_workspace_bytes(const dpsgd_layer* layers, int32_t n) {
  int64_t partials = 0;
  for (int32_t base = 0; base < n; base += kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    partials += norm_wgs(args_of(layers + base, m, nullptr, nullptr));
  }
  return (size_t)partials * sizeof(double);
}

int launch_global_clip(const dpsgd_layer* layers, int32_t n, const float* const* grads,
                       float* const* outs, float max_norm, float* norm_out, float* factor_out,
                       void* workspace, hipStream_t stream) {
  // The scaling has a workgroup a block; launches that cannot be made are refused
  // before the first.
  for (int32_t base = 0; outs && base < n; base += kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    if (!launchable(args_of(layers + base, m, nullptr, nullptr).blocks, kThreads))
      return DPSGD_ERR_INVALID_ARG;
  }
  double* partials = static_cast<double*>(workspace);
  int64_t at = 0;
  for (int32_t base = 0; base < n; base += kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    ClipArgs a = args_of(layers + base, m, grads + base, nullptr);
    a.partials = partials + at;
    hipLaunchKernelGGL(sum_squares_kernel, dim3((uint32_t)norm_wgs(a)), dim3(kThreads), 0, stream, a);
    at += norm_wgs(a);
  }
  if (!outs) {
    ClipArgs a{};
    a.all = partials;
    a.n_all = at;
    a.norm_out = norm_out;
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, stream, a);
    return check_launch();
  }
  // Launches in reverse, for the same reason as the blocks of one.
  int64_t apart = 0;
  for (int32_t l = 0; l < n; ++l)
    if (outs[l] != grads[l]) apart += layers[l].d_in * layers[l].d_out * (int64_t)sizeof(float);
  const int32_t last = (n - 1) / kMaxLayersPerLaunch * kMaxLayersPerLaunch;
  for (int32_t base = last; base >= 0; base -= kMaxLayersPerLaunch) {
    const int32_t m = n - base < kMaxLayersPerLaunch ? n - base : kMaxLayersPerLaunch;
    ClipArgs a = args_of(layers + base, m, grads + base, outs + base);
    a.all = partials;
    a.n_all = at;
    a.max_norm = max_norm;
    if (base == last) {
      a.norm_out = norm_out;
      a.factor_out = factor_out;
    }
    const dim3 grid((uint32_t)a.blocks);
    if (apart >= kPastCaches)
      hipLaunchKernelGGL(scale_kernel<true>, grid, dim3(kThreads), 0, stream, a);
    else
      hipLaunchKernelGGL(scale_kernel<false>, grid, dim3(kThreads), 0, stream, a);
  }
  return check_launch();
}

}  // namespace dpsgd
