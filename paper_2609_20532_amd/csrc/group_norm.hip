// Group norm over channels-last rows x [B][S][C], with an activation, and its
// gradients.
//
//   xh = (x - mu) rstd,  z = gamma xh + beta,  y = act(z)
//   dz = dy act'(z);  per example: dbeta_i = sum_s dz, dgamma_i = sum_s dz xh
//   dx = rstd (gamma dz - m1 - xh m2),  m1 = mean(gamma dz), m2 = mean(gamma dz xh)
//
// with mu, rstd, m1 and m2 per example and group of C / groups neighbouring
// channels. Both directions sum over the positions channel by channel (a
// thread keeps a fixed set of channels, so that any group width works), which
// for the gradient are dgamma_i and dbeta_i themselves, and then over the
// channels of a group. The statistics are means and sums of squared deviations
// (no difference of large sums): each thread takes eight rows at a time, in two
// passes over registers, and results are merged by their counts.
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

constexpr float kGelu0 = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGelu1 = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == DPSGD_ACT_RELU) return z < 0.0f ? 0.0f : z;   // a NaN stays
  if constexpr (ACT == DPSGD_ACT_SILU) return z / (1.0f + expf(-z));
  if constexpr (ACT == DPSGD_ACT_GELU) {
    const float u = kGelu0 * fmaf(kGelu1 * z * z, z, z);
    return z / (1.0f + expf(-2.0f * u));   // 0.5 z (1 + tanh u)
  }
  return z;
}

// act'(z).
template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
  if constexpr (ACT == DPSGD_ACT_RELU) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
  if constexpr (ACT == DPSGD_ACT_SILU) {
    const float p = 1.0f / (1.0f + expf(-z));
    return p * fmaf(z, 1.0f - p, 1.0f);
  }
  if constexpr (ACT == DPSGD_ACT_GELU) {
    const float u = kGelu0 * fmaf(kGelu1 * z * z, z, z);
    const float p = 1.0f / (1.0f + expf(-2.0f * u));
    const float du = kGelu0 * fmaf(3.0f * kGelu1 * z, z, 1.0f);
    return p + 2.0f * z * p * (1.0f - p) * du;
  }
  return 1.0f;
}

struct GnArgs {
  const void* x;
  const void* dy;
  void* out;             // y or dx
  const float* gamma;    // NULL: 1
  const float* beta;     // NULL: 0
  float* mean;           // [B][groups]
  float* rstd;
  float* dgamma;         // [B][C]
  float* dbeta;
  float* partials;       // [B][chunks][C][3]: a channel's Stat (backward: [2], its sums)
  float2* sums;          // [B][groups] m1, m2
  int64_t S;
  int64_t rows;          // rows of a chunk
  int32_t B, C, groups, width;
  int32_t chunks, blocks;   // chunks of an example's rows, blocks of its channels
  int32_t units;         // channel vectors of a block
  float eps;
};

// Where a workgroup of the passes over the rows is.
struct Place {
  int64_t b, r0, r1;
  int32_t chunk, c, r, step;   // first channel, first row and row step of the thread
  bool active;
};

template <int V>
__device__ __forceinline__ Place place_of(const GnArgs& a) {
  Place p;
  const int64_t w = blockIdx.x;
  const int32_t blk = (int32_t)(w % a.blocks);
  p.chunk = (int32_t)(w / a.blocks % a.chunks);
  p.b = w / a.blocks / a.chunks;
  p.step = kThreads / a.units;
  p.r = threadIdx.x / a.units;
  p.c = (blk * a.units + threadIdx.x % a.units) * V;
  p.active = p.r < p.step && p.c < a.C;
  p.r0 = p.chunk * a.rows;
  p.r1 = p.r0 + a.rows < a.S ? p.r0 + a.rows : a.S;
  return p;
}

// n values: their mean as an unevaluated sum hi + lo (lo at most a rounding of
// hi), and the sum of squared deviations from it. The second word keeps the
// difference of two means, whose square enters the sum when they are merged, as
// exact as the values themselves when the mean is far larger than the spread.
struct Stat {
  float n, hi, lo, m2;
};

__device__ __forceinline__ void merge(Stat& a, const Stat& b) {
  const float t = a.n + b.n;
  if (t == 0.0f) return;
  const float w = b.n / t, d = (b.hi - a.hi) + (b.lo - a.lo);
  a.m2 = a.m2 + b.m2 + d * d * a.n * w;
  const float lo = fmaf(d, w, a.lo), hi = a.hi + lo;
  const float back = hi - a.hi;
  a.lo = (a.hi - (hi - back)) + (lo - back);
  a.hi = hi;
  a.n = t;
}

template <class T, int V>
__global__ __launch_bounds__(kThreads) void gn_stats_kernel(GnArgs a) {
  __shared__ float lds[kThreads][3 * V + 1];
  const Place p = place_of<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.b * a.S * a.C + p.c;
  Stat st[V] = {};
  if (p.active) {
    for (int64_t r = p.r0 + p.r; r < p.r1; r += 8 * p.step) {
      float v[8][V];
      int m = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t at = r + k * p.step;
        if (at < p.r1) {
          load_vec<V>(x + at * a.C, v[k]);
          m = k + 1;
        } else {
#pragma unroll
          for (int c = 0; c < V; ++c) v[k][c] = 0.0f;
        }
      }
      const float n = (float)m;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        float s = 0.0f, e = 0.0f, q = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k][c];
        s /= n;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float d = k < m ? v[k][c] - s : 0.0f;
          e += d;
          q = fmaf(d, d, q);
        }
        e /= n;
        merge(st[c], Stat{n, s, e, fmaf(-n * e, e, q)});
      }
    }
  }
  float* mine = lds[threadIdx.x];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    mine[3 * c] = st[c].hi;
    mine[3 * c + 1] = st[c].lo;
    mine[3 * c + 2] = st[c].m2;
  }
  mine[3 * V] = st[0].n;
  int half = 1;
  while (half < p.step) half <<= 1;
  for (half >>= 1; half >= 1; half >>= 1) {
    __syncthreads();
    if (p.active && p.r < half && p.r + half < p.step) {
      const float* other = lds[threadIdx.x + half * a.units];
#pragma unroll
      for (int c = 0; c < V; ++c) {
        merge(st[c], Stat{other[3 * V], other[3 * c], other[3 * c + 1], other[3 * c + 2]});
        mine[3 * c] = st[c].hi;
        mine[3 * c + 1] = st[c].lo;
        mine[3 * c + 2] = st[c].m2;
      }
      mine[3 * V] = st[0].n;
    }
  }
  if (p.active && p.r == 0) {
    float* out = a.partials + ((p.b * a.chunks + p.chunk) * a.C + p.c) * 3;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      out[3 * c] = st[c].hi;
      out[3 * c + 1] = st[c].lo;
      out[3 * c + 2] = st[c].m2;
    }
  }
}

// One wave per example and group: its chunks' and channels' statistics merged.
__global__ __launch_bounds__(kThreads) void gn_finish_kernel(GnArgs a) {
  const int64_t job = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (job >= (int64_t)a.B * a.groups) return;
  const int64_t b = job / a.groups, g = job - b * a.groups;
  Stat st{};
  const int64_t items = (int64_t)a.chunks * a.width;
  for (int64_t k = lane; k < items; k += 64) {
    const int64_t chunk = k / a.width;
    const float* s = a.partials + ((b * a.chunks + chunk) * a.C + g * a.width + (k - chunk * a.width)) * 3;
    const int64_t left = a.S - chunk * a.rows;
    merge(st, Stat{(float)(left < a.rows ? left : a.rows), s[0], s[1], s[2]});
  }
  for (int off = 32; off >= 1; off >>= 1) {
    const Stat other{__shfl_down(st.n, off, 64), __shfl_down(st.hi, off, 64),
                     __shfl_down(st.lo, off, 64), __shfl_down(st.m2, off, 64)};
    if (lane < off) merge(st, other);
  }
  if (lane == 0) {
    a.mean[job] = st.hi;
    a.rstd[job] = 1.0f / sqrtf(st.m2 / ((float)a.S * (float)a.width) + a.eps);
  }
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void gn_apply_kernel(GnArgs a) {
  const Place p = place_of<V>(a);
  if (!p.active) return;
  const T* x = static_cast<const T*>(a.x) + p.b * a.S * a.C + p.c;
  T* y = static_cast<T*>(a.out) + p.b * a.S * a.C + p.c;
  float mu[V], rs[V], ga[V], be[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int64_t g = p.b * a.groups + (p.c + c) / a.width;
    mu[c] = a.mean[g];
    rs[c] = a.rstd[g];
    ga[c] = a.gamma ? a.gamma[p.c + c] : 1.0f;
    be[c] = a.beta ? a.beta[p.c + c] : 0.0f;
  }
  for (int64_t r = p.r0 + p.r; r < p.r1; r += p.step) {
    float v[V];
    load_vec<V>(x + r * a.C, v);
#pragma unroll
    for (int c = 0; c < V; ++c) v[c] = act_of<ACT>(fmaf((v[c] - mu[c]) * rs[c], ga[c], be[c]));
    store_vec<V>(y + r * a.C, v);
  }
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void gn_grad_sums_kernel(GnArgs a) {
  __shared__ float lds[kThreads][2 * V + 1];
  const Place p = place_of<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.b * a.S * a.C + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.b * a.S * a.C + p.c;
  float sb[V] = {}, sg[V] = {};
  if (p.active) {
    float mu[V], rs[V], ga[V], be[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int64_t g = p.b * a.groups + (p.c + c) / a.width;
      mu[c] = a.mean[g];
      rs[c] = a.rstd[g];
      ga[c] = a.gamma ? a.gamma[p.c + c] : 1.0f;
      be[c] = a.beta ? a.beta[p.c + c] : 0.0f;
    }
    for (int64_t r = p.r0 + p.r; r < p.r1; r += p.step) {
      float v[V], d[V];
      load_vec<V>(x + r * a.C, v);
      load_vec<V>(dy + r * a.C, d);
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float xh = (v[c] - mu[c]) * rs[c];
        const float dz = d[c] * slope_of<ACT>(fmaf(xh, ga[c], be[c]));
        sb[c] += dz;
        sg[c] = fmaf(dz, xh, sg[c]);
      }
    }
  }
  float* mine = lds[threadIdx.x];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    mine[2 * c] = sb[c];
    mine[2 * c + 1] = sg[c];
  }
  int half = 1;
  while (half < p.step) half <<= 1;
  for (half >>= 1; half >= 1; half >>= 1) {
    __syncthreads();
    if (p.active && p.r < half && p.r + half < p.step) {
      const float* other = lds[threadIdx.x + half * a.units];
#pragma unroll
      for (int c = 0; c < 2 * V; ++c) mine[c] += other[c];
    }
  }
  if (p.active && p.r == 0) {
    float* out = a.partials + ((p.b * a.chunks + p.chunk) * a.C + p.c) * 2;
#pragma unroll
    for (int c = 0; c < 2 * V; ++c) out[c] = mine[c];
  }
}

// One wave per example and group: dgamma_i and dbeta_i of its channels, and the
// means m1 and m2.
__global__ __launch_bounds__(kThreads) void gn_grad_finish_kernel(GnArgs a) {
  const int64_t job = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (job >= (int64_t)a.B * a.groups) return;
  const int64_t b = job / a.groups, g = job - b * a.groups;
  float s1 = 0.0f, s2 = 0.0f;
  for (int32_t k = lane; k < a.width; k += 64) {
    const int64_t c = g * a.width + k;
    float sb = 0.0f, sg = 0.0f;
    for (int32_t chunk = 0; chunk < a.chunks; ++chunk) {
      const float* s = a.partials + ((b * a.chunks + chunk) * a.C + c) * 2;
      sb += s[0];
      sg += s[1];
    }
    a.dbeta[b * a.C + c] = sb;
    a.dgamma[b * a.C + c] = sg;
    const float ga = a.gamma ? a.gamma[c] : 1.0f;
    s1 = fmaf(ga, sb, s1);
    s2 = fmaf(ga, sg, s2);
  }
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  const float inv = 1.0f / ((float)a.S * (float)a.width);
  if (lane == 0) a.sums[job] = make_float2(s1 * inv, s2 * inv);
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void gn_grad_apply_kernel(GnArgs a) {
  const Place p = place_of<V>(a);
  if (!p.active) return;
  const T* x = static_cast<const T*>(a.x) + p.b * a.S * a.C + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.b * a.S * a.C + p.c;
  T* dx = static_cast<T*>(a.out) + p.b * a.S * a.C + p.c;
  float mu[V], rs[V], ga[V], be[V], m1[V], m2[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int64_t g = p.b * a.groups + (p.c + c) / a.width;
    mu[c] = a.mean[g];
    rs[c] = a.rstd[g];
    ga[c] = a.gamma ? a.gamma[p.c + c] : 1.0f;
    be[c] = a.beta ? a.beta[p.c + c] : 0.0f;
    m1[c] = a.sums[g].x;
    m2[c] = a.sums[g].y;
  }
  for (int64_t r = p.r0 + p.r; r < p.r1; r += p.step) {
    float v[V], d[V];
    load_vec<V>(x + r * a.C, v);
    load_vec<V>(dy + r * a.C, d);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const float xh = (v[c] - mu[c]) * rs[c];
      const float dz = d[c] * slope_of<ACT>(fmaf(xh, ga[c], be[c]));
      d[c] = rs[c] * (fmaf(dz, ga[c], -m1[c]) - xh * m2[c]);
    }
    store_vec<V>(dx + r * a.C, d);
  }
}

// Split of the passes over the rows: blocks of channel vectors, and chunks of
// rows so that about 2048 workgroups run, each thread with at least eight rows.
struct GnPlan {
  int vec, units, blocks;
  int64_t chunks, rows;
};

GnPlan plan_of(const dpsgd_group_norm& n) {
  GnPlan p;
  p.vec = vec_width(n.C, n.dtype == DPSGD_BF16 ? 8 : 4);
  const int64_t units = n.C / p.vec;
  p.blocks = (int)ceil_div(units, kThreads);
  p.units = (int)ceil_div(units, p.blocks);
  const int64_t least = 8 * (kThreads / p.units);
  int64_t chunks = ceil_div(2048, n.B * p.blocks);
  const int64_t most = ceil_div(n.S, least);
  if (chunks > most) chunks = most;
  p.rows = ceil_div(n.S, chunks);
  p.chunks = ceil_div(n.S, p.rows);
  return p;
}

size_t stat_bytes(const dpsgd_group_norm& n) {
  return round_up((size_t)(n.B * n.groups) * sizeof(float), 256);
}

GnArgs args_of(const dpsgd_group_norm& n, const GnPlan& p, const void* x, void* out, void* ws) {
  GnArgs a{};
  a.x = x;
  a.out = out;
  a.gamma = n.gamma;
  a.beta = n.beta;
  a.mean = static_cast<float*>(ws);
  a.rstd = reinterpret_cast<float*>(static_cast<char*>(ws) + stat_bytes(n));
  a.sums = static_cast<float2*>(ws);   // the backward pass is given mean and rstd
  a.partials = reinterpret_cast<float*>(static_cast<char*>(ws) + 2 * stat_bytes(n));
  a.S = n.S;
  a.rows = p.rows;
  a.B = (int32_t)n.B;
  a.C = (int32_t)n.C;
  a.groups = (int32_t)n.groups;
  a.width = (int32_t)(n.C / n.groups);
  a.chunks = (int32_t)p.chunks;
  a.blocks = p.blocks;
  a.units = p.units;
  a.eps = n.eps;
  return a;
}

template <class T, int V, int ACT>
int run_forward(const GnArgs& a, uint32_t wgs, uint32_t finish, hipStream_t stream) {
  hipLaunchKernelGGL((gn_stats_kernel<T, V>), dim3(wgs), dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(gn_finish_kernel, dim3(finish), dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL((gn_apply_kernel<T, V, ACT>), dim3(wgs), dim3(kThreads), 0, stream, a);
  return check_launch();
}

template <class T, int V, int ACT>
int run_backward(const GnArgs& a, uint32_t wgs, uint32_t finish, hipStream_t stream) {
  hipLaunchKernelGGL((gn_grad_sums_kernel<T, V, ACT>), dim3(wgs), dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(gn_grad_finish_kernel, dim3(finish), dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL((gn_grad_apply_kernel<T, V, ACT>), dim3(wgs), dim3(kThreads), 0, stream, a);
  return check_launch();
}

template <class T, int V>
int run_act(int act, bool backward, const GnArgs& a, uint32_t wgs, uint32_t finish,
            hipStream_t stream) {
  switch (act) {
#define DPSGD_ACT(A)                                                      \
  case A:                                                                 \
    return backward ? run_backward<T, V, A>(a, wgs, finish, stream)       \
                    : run_forward<T, V, A>(a, wgs, finish, stream);
    DPSGD_ACT(DPSGD_ACT_RELU)
    DPSGD_ACT(DPSGD_ACT_SILU)
    DPSGD_ACT(DPSGD_ACT_GELU)
    DPSGD_ACT(DPSGD_ACT_NONE)
#undef DPSGD_ACT
    default: return DPSGD_ERR_UNSUPPORTED;
  }
}

int run_group_norm(const dpsgd_group_norm& n, const GnPlan& p, bool backward, const GnArgs& a,
                   hipStream_t stream) {
  const int64_t wgs = n.B * p.chunks * p.blocks, finish = ceil_div(n.B * n.groups, kThreads / 64);
  if (wgs > 0x7FFFFFFF || finish > 0x7FFFFFFF) return DPSGD_ERR_INVALID_ARG;
  const uint32_t w = (uint32_t)wgs, f = (uint32_t)finish;
  if (n.dtype == DPSGD_BF16) {
    switch (p.vec) {
      case 8: return run_act<uint16_t, 8>(n.act, backward, a, w, f, stream);
      case 4: return run_act<uint16_t, 4>(n.act, backward, a, w, f, stream);
      case 2: return run_act<uint16_t, 2>(n.act, backward, a, w, f, stream);
      default: return run_act<uint16_t, 1>(n.act, backward, a, w, f, stream);
    }
  }
  switch (p.vec) {
    case 4: return run_act<float, 4>(n.act, backward, a, w, f, stream);
    case 2: return run_act<float, 2>(n.act, backward, a, w, f, stream);
    default: return run_act<float, 1>(n.act, backward, a, w, f, stream);
  }
}

}  // namespace

// Workspace: mean and rstd where the caller does not take them (backward: m1 and
// m2), then the chunks' statistics of every channel.
size_t group_norm_workspace_bytes(const dpsgd_group_norm& n) {
  const GnPlan p = plan_of(n);
  return 2 * stat_bytes(n) + (size_t)(n.B * p.chunks * n.C) * 3 * sizeof(float);
}

int launch_group_norm_forward(const dpsgd_group_norm& n, const void* x, void* y, float* mean,
                              float* rstd, void* workspace, hipStream_t stream) {
  const GnPlan p = plan_of(n);
  GnArgs a = args_of(n, p, x, y, workspace);
  if (mean) a.mean = mean;
  if (rstd) a.rstd = rstd;
  return run_group_norm(n, p, false, a, stream);
}

int launch_group_norm_backward(const dpsgd_group_norm& n, const void* x, const void* dy,
                               const float* mean, const float* rstd, void* dx, float* dgamma,
                               float* dbeta, void* workspace, hipStream_t stream) {
  const GnPlan p = plan_of(n);
  GnArgs a = args_of(n, p, x, dx, workspace);
  a.dy = dy;
  a.mean = const_cast<float*>(mean);   // read only in the backward kernels
  a.rstd = const_cast<float*>(rstd);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  return run_group_norm(n, p, true, a, stream);
}

}  // namespace dpsgd
