// Gaussian noise of the DP-SGD step: Philox4x32-10 + Box-Muller, added in place.
//
// Paper: Section 2.2, z_t ~ N(0, sigma^2 C^2 I) added to the clipped sum and
// scaled by 1/|B_t|; GPU-side algorithm, noise step. The generator is
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC'11) with the Box-Muller (1958)
// transform; the paper does not fix one.
//
// The pass is bound by HBM traffic (read + write of 4 bytes per element) and,
// close behind, by integer/transcendental ALU work: one Philox block (ten
// rounds, two 32x32->64 products each) and two log/sqrt/sin/cos sets per four
// elements. Each thread owns whole 16-byte blocks so loads and stores are
// 16-byte, fully coalesced, and every launch covers all tensors of the call.
#include <math.h>

#include "philox.h"

namespace dpsgd {
namespace {

struct NoiseSeg {
  float* ptr;
  int64_t numel;
  uint32_t tensor_id;
  uint32_t wg_begin;   // first workgroup of this tensor in the launch
  uint32_t aligned;    // ptr is 16-byte aligned
  uint32_t pad;
};

struct NoiseArgs {
  NoiseSeg seg[kMaxLayersPerLaunch];
  int n_seg;
  uint32_t k0, k1, step;
  float sigmaC, scale;
};

constexpr int kBlocksPerThread = 4;
constexpr int kBlocksPerWG = kThreads * kBlocksPerThread;

__global__ __launch_bounds__(kThreads) void noise_kernel(NoiseArgs args) {
  // Segment of this workgroup: binary search over wg_begin (uniform).
  int lo = 0, hi = args.n_seg - 1;
  const uint32_t wg = blockIdx.x;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (args.seg[mid].wg_begin <= wg) lo = mid; else hi = mid - 1;
  }
  const NoiseSeg s = args.seg[lo];
  const int64_t first_block = (int64_t)(wg - s.wg_begin) * kBlocksPerWG;
  const int64_t n_blocks = (s.numel + 3) >> 2;
  const float sc = args.scale, sgc = args.sigmaC;
  const bool with_noise = sgc != 0.0f;

#pragma unroll
  for (int u = 0; u < kBlocksPerThread; ++u) {
    const int64_t j = first_block + (int64_t)u * kThreads + threadIdx.x;
    if (j >= n_blocks) break;
    float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
    if (with_noise) z = normals_of_block((uint64_t)j, s.tensor_id, args.step, args.k0, args.k1);
    const int64_t e0 = j * 4;
    if (s.aligned && e0 + 4 <= s.numel) {
      float4* p = reinterpret_cast<float4*>(s.ptr + e0);
      float4 g = *p;
      g.x = sc * fmaf(sgc, z.x, g.x);
      g.y = sc * fmaf(sgc, z.y, g.y);
      g.z = sc * fmaf(sgc, z.z, g.z);
      g.w = sc * fmaf(sgc, z.w, g.w);
      *p = g;
    } else {
      const float zz[4] = {z.x, z.y, z.z, z.w};
      for (int w = 0; w < 4; ++w) {
        if (e0 + w < s.numel) {
          float* p = s.ptr + e0 + w;
          *p = sc * fmaf(sgc, zz[w], *p);
        }
      }
    }
  }
}

__global__ __launch_bounds__(kThreads) void philox_u32_kernel(uint32_t* out, int64_t first_block,
                                                              int64_t n_blocks, uint32_t k0,
                                                              uint32_t k1, uint32_t tensor_id,
                                                              uint32_t step) {
  const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (b >= n_blocks) return;
  const uint64_t j = (uint64_t)(first_block + b);
  const uint4 w = philox4x32_10((uint32_t)j, (uint32_t)(j >> 32), tensor_id, step, k0, k1);
  out[4 * b + 0] = w.x;
  out[4 * b + 1] = w.y;
  out[4 * b + 2] = w.z;
  out[4 * b + 3] = w.w;
}

__global__ __launch_bounds__(kThreads) void gaussian_kernel(float* out, int64_t n, uint32_t k0,
                                                            uint32_t k1, uint32_t tensor_id,
                                                            uint32_t step) {
  const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t e0 = j * 4;
  if (e0 >= n) return;
  const float4 z = normals_of_block((uint64_t)j, tensor_id, step, k0, k1);
  const float zz[4] = {z.x, z.y, z.z, z.w};
  for (int w = 0; w < 4; ++w)
    if (e0 + w < n) out[e0 + w] = zz[w];
}

// ------------------------------------------------------- noise + AdamW step

struct AdamSeg {
  const float* grad;   // clipped sum S (read only)
  float* param;
  float* m;
  float* v;
  float* noisy;        // optional output of the noisy gradient (nullptr: not written)
  int64_t numel;
  uint32_t tensor_id;
  uint32_t wg_begin;
};

struct AdamArgs {
  AdamSeg seg[kMaxLayersPerLaunch];
  int n_seg;
  uint32_t k0, k1, step;
  float sigmaC, scale;
  float beta1, beta2, one_m_beta1, one_m_beta2;
  float step_size;      // lr / (1 - beta1^t)
  float inv_sqrt_bc2;   // 1 / sqrt(1 - beta2^t)
  float eps;
  float decay;          // 1 - lr * weight_decay
};

// One element of the update: g = scale (S + sigma C z); moments; decoupled
// decay and the bias-corrected step (appendix "One-step AdamW map").
__device__ __forceinline__ void adamw_elem(const AdamArgs& a, float S, float z, float& p, float& m,
                                           float& v, float& g) {
  g = a.scale * fmaf(a.sigmaC, z, S);
  m = fmaf(a.beta1, m, a.one_m_beta1 * g);
  v = fmaf(a.beta2, v, a.one_m_beta2 * (g * g));
  const float denom = fmaf(sqrtf(v), a.inv_sqrt_bc2, a.eps);
  p = fmaf(p, a.decay, -a.step_size * (m / denom));
}

// 16-byte streaming load/store: the lines are not kept in the caches, since
// every byte of the optimizer pass is touched exactly once (measured 9% faster
// than plain accesses on cold parameters and moments).
__device__ __forceinline__ f32x4_t ld_stream(const float* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p));
}

__device__ __forceinline__ void st_stream(f32x4_t x, float* p) {
  __builtin_nontemporal_store(x, reinterpret_cast<f32x4_t*>(p));
}

__global__ __launch_bounds__(kThreads) void noise_adamw_kernel(AdamArgs args) {
  int lo = 0, hi = args.n_seg - 1;
  const uint32_t wg = blockIdx.x;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (args.seg[mid].wg_begin <= wg) lo = mid; else hi = mid - 1;
  }
  const AdamSeg& s = args.seg[lo];
  const int64_t first_block = (int64_t)(wg - s.wg_begin) * kBlocksPerWG;
  const int64_t n_blocks = (s.numel + 3) >> 2;
  const bool with_noise = args.sigmaC != 0.0f;

  if ((first_block + kBlocksPerWG) * 4 <= s.numel) {
    // Whole workgroup in range: issue every load of the thread's blocks
    // before any arithmetic, so 16 independent 16-byte loads are in flight
    // while the Philox rounds run (every pointer is 16-byte aligned, checked
    // by the API).
    f32x4_t S[kBlocksPerThread], p[kBlocksPerThread], m[kBlocksPerThread], v[kBlocksPerThread];
#pragma unroll
    for (int u = 0; u < kBlocksPerThread; ++u) {
      const int64_t e0 = (first_block + (int64_t)u * kThreads + threadIdx.x) * 4;
      S[u] = ld_stream(s.grad + e0);
      p[u] = ld_stream(s.param + e0);
      m[u] = ld_stream(s.m + e0);
      v[u] = ld_stream(s.v + e0);
    }
#pragma unroll
    for (int u = 0; u < kBlocksPerThread; ++u) {
      const int64_t j = first_block + (int64_t)u * kThreads + threadIdx.x;
      float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
      if (with_noise) z = normals_of_block((uint64_t)j, s.tensor_id, args.step, args.k0, args.k1);
      const float zz[4] = {z.x, z.y, z.z, z.w};
      f32x4_t g;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float pc = p[u][c], mc = m[u][c], vc = v[u][c], gc;
        adamw_elem(args, S[u][c], zz[c], pc, mc, vc, gc);
        p[u][c] = pc;
        m[u][c] = mc;
        v[u][c] = vc;
        g[c] = gc;
      }
      const int64_t e0 = j * 4;
      st_stream(p[u], s.param + e0);
      st_stream(m[u], s.m + e0);
      st_stream(v[u], s.v + e0);
      if (s.noisy) st_stream(g, s.noisy + e0);
    }
    return;
  }

  // Last workgroup of a tensor: block by block, scalar past the last whole block.
  for (int u = 0; u < kBlocksPerThread; ++u) {
    const int64_t j = first_block + (int64_t)u * kThreads + threadIdx.x;
    if (j >= n_blocks) break;
    float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
    if (with_noise) z = normals_of_block((uint64_t)j, s.tensor_id, args.step, args.k0, args.k1);
    const float zz[4] = {z.x, z.y, z.z, z.w};
    for (int w = 0; w < 4; ++w) {
      const int64_t e = j * 4 + w;
      if (e >= s.numel) break;
      float p = s.param[e], m = s.m[e], v = s.v[e], g;
      adamw_elem(args, s.grad[e], zz[w], p, m, v, g);
      s.param[e] = p;
      s.m[e] = m;
      s.v[e] = v;
      if (s.noisy) s.noisy[e] = g;
    }
  }
}

}  // namespace

int launch_noise(const dpsgd_layer* layers, int n_layers, float* const* grads, float sigma,
                 float C, uint64_t seed, uint32_t step, float scale, hipStream_t stream) {
  for (int base = 0; base < n_layers; base += kMaxLayersPerLaunch) {
    const int n = n_layers - base < kMaxLayersPerLaunch ? n_layers - base : kMaxLayersPerLaunch;
    NoiseArgs args{};
    args.n_seg = n;
    args.k0 = (uint32_t)seed;
    args.k1 = (uint32_t)(seed >> 32);
    args.step = step;
    args.sigmaC = sigma * C;
    args.scale = scale;
    int64_t wgs = 0;
    for (int l = 0; l < n; ++l) {
      const dpsgd_layer& L = layers[base + l];
      NoiseSeg& s = args.seg[l];
      s.ptr = grads[base + l];
      s.numel = L.d_out * L.d_in;
      s.tensor_id = L.tensor_id;
      s.wg_begin = (uint32_t)wgs;
      s.aligned = aligned16(s.ptr) ? 1u : 0u;
      wgs += ceil_div(ceil_div(s.numel, 4), kBlocksPerWG);
    }
    if (wgs <= 0) continue;
    if (wgs > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
    hipLaunchKernelGGL(noise_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, args);
    if (check_launch() != DPSGD_OK) return DPSGD_ERR_HIP;
  }
  return DPSGD_OK;
}

int launch_philox_u32(uint32_t* out, int64_t first_block, int64_t n_blocks, uint64_t seed,
                      uint32_t tensor_id, uint32_t step, hipStream_t stream) {
  const int64_t wgs = ceil_div(n_blocks, kThreads);
  if (wgs > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
  hipLaunchKernelGGL(philox_u32_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, out,
                     first_block, n_blocks, (uint32_t)seed, (uint32_t)(seed >> 32), tensor_id, step);
  return check_launch();
}

int launch_gaussian(float* out, int64_t n, uint64_t seed, uint32_t tensor_id, uint32_t step,
                    hipStream_t stream) {
  const int64_t wgs = ceil_div(ceil_div(n, 4), kThreads);
  if (wgs > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
  hipLaunchKernelGGL(gaussian_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, out, n,
                     (uint32_t)seed, (uint32_t)(seed >> 32), tensor_id, step);
  return check_launch();
}

int launch_noise_adamw(const dpsgd_layer* layers, int n_layers, const float* const* grads,
                       float* const* params, float* const* ms, float* const* vs,
                       float* const* noisy, float sigma, float C, uint64_t seed, uint32_t step,
                       float scale, const dpsgd_adamw& opt, hipStream_t stream) {
  const double bc1 = 1.0 - pow((double)opt.beta1, (double)opt.t);
  const double bc2 = 1.0 - pow((double)opt.beta2, (double)opt.t);
  for (int base = 0; base < n_layers; base += kMaxLayersPerLaunch) {
    const int n = n_layers - base < kMaxLayersPerLaunch ? n_layers - base : kMaxLayersPerLaunch;
    AdamArgs args{};
    args.n_seg = n;
    args.k0 = (uint32_t)seed;
    args.k1 = (uint32_t)(seed >> 32);
    args.step = step;
    args.sigmaC = sigma * C;
    args.scale = scale;
    args.beta1 = opt.beta1;
    args.beta2 = opt.beta2;
    args.one_m_beta1 = (float)(1.0 - (double)opt.beta1);
    args.one_m_beta2 = (float)(1.0 - (double)opt.beta2);
    args.step_size = (float)((double)opt.lr / bc1);
    args.inv_sqrt_bc2 = (float)(1.0 / sqrt(bc2));
    args.eps = opt.eps;
    args.decay = (float)(1.0 - (double)opt.lr * (double)opt.weight_decay);
    int64_t wgs = 0;
    for (int l = 0; l < n; ++l) {
      const dpsgd_layer& L = layers[base + l];
      AdamSeg& sg = args.seg[l];
      sg.grad = grads[base + l];
      sg.param = params[base + l];
      sg.m = ms[base + l];
      sg.v = vs[base + l];
      sg.noisy = noisy ? noisy[base + l] : nullptr;
      sg.numel = L.d_out * L.d_in;
      sg.tensor_id = L.tensor_id;
      sg.wg_begin = (uint32_t)wgs;
      wgs += ceil_div(ceil_div(sg.numel, 4), kBlocksPerWG);
    }
    if (wgs <= 0) continue;
    if (wgs > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
    hipLaunchKernelGGL(noise_adamw_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, args);
    if (check_launch() != DPSGD_OK) return DPSGD_ERR_HIP;
  }
  return DPSGD_OK;
}

}  // namespace dpsgd
