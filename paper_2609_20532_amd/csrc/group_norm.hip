// Group norm over channels-last rows x [B][S][C], with an activation, and its
// gradients.
//
//   xh = (x - mu) rstd,  z = gamma xh + beta,  y = act(z)
//   dz = dy act'(z);  per example: dbeta_i = sum_s dz, dgamma_i = sum_s dz xh
//   dx = rstd (gamma dz - m1 - xh m2),  m1 = mean(gamma dz), m2 = mean(gamma dz xh)
//
// with mu, rstd, m1 and m2 per example and group of C / groups neighbouring
// channels. Bound by memory traffic. A workgroup takes a tile, some rows and a
// block of channels of one example, into registers; a thread keeps a fixed set of
// channels, so that any group width works. Where all rows of whole groups fit one
// tile, x (and dy) are read once, and the result is written from the registers
// in the same launch. Otherwise a first pass leaves the tiles' statistics, a
// second one joins them, and a third reads x (and dy) again, from the last-level
// cache where it holds them.
//
// [256, 1024, 64]: float32 forward 33-37 us (134 MB, 3.9 TB/s: all tiles load, then
// all store), backward 37 us (201 MB, 5.4 TB/s); bf16 forward 20 us (67 MB).
// [2, 16384, 320] in bf16, which has no tile of all rows: forward 11 + 4 + 12 us,
// backward 15 + 4 + 14, mostly each tile's sums and the launches.
//
// Statistics are taken in two passes over the registers, the mean and then the
// deviations from it, and tiles are merged by their counts: no difference of
// large sums is formed.
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

constexpr int kTile = 1024;    // most threads of a tile's workgroup
constexpr int kPartTile = 256; // threads of a tile that has a part of the rows or of a group
constexpr uint32_t kXcds = 8;
constexpr int kGradRows = 8;   // rows of a thread in a backward tile

// Rows of a thread in a forward tile: 32 registers of 4 elements each.
template <class T>
constexpr int kTileRows = 32 / (int)sizeof(T);

// 1 / (1 + exp(-z)) by the hardware's exponential and reciprocal. The exponent's
// rounding enters the exponential times |z|: the relative error is at most
// (1.25 |z| + 7) 2^-24 for z < 0 (z sigmoid(z) measured, in 2^-23: 1.4 from -1 on
// up, 4.7 at -10 .. -8, 15 at -30 .. -20, 32 at -80 .. -60), and the value is 0
// from about -87 on, where it would be below 2e-38.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}

constexpr float kGelu0 = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGelu1 = 0.044715f;

// x = act(x), or slope = act'(z), for V values. 0.5 (1 + tanh u) = sigmoid(2 u).
template <int ACT, int V>
__device__ __forceinline__ void activate(float (&x)[V]) {
#pragma unroll
  for (int c = 0; c < V; ++c) {
    if constexpr (ACT == DPSGD_ACT_RELU) x[c] = x[c] < 0.0f ? 0.0f : x[c];   // a NaN stays
    if constexpr (ACT == DPSGD_ACT_SILU) x[c] *= sigmoid(x[c]);
    if constexpr (ACT == DPSGD_ACT_GELU)
      x[c] *= sigmoid(2.0f * kGelu0 * fmaf(kGelu1 * x[c] * x[c], x[c], x[c]));
  }
}

template <int ACT, int V>
__device__ __forceinline__ void slopes(const float (&z)[V], float (&slope)[V]) {
#pragma unroll
  for (int c = 0; c < V; ++c) {
    slope[c] = 1.0f;
    if constexpr (ACT == DPSGD_ACT_RELU) slope[c] = z[c] > 0.0f ? 1.0f : (z[c] == z[c] ? 0.0f : z[c]);
    if constexpr (ACT == DPSGD_ACT_SILU) {
      const float p = sigmoid(z[c]);
      slope[c] = p * fmaf(z[c], 1.0f - p, 1.0f);
    }
    if constexpr (ACT == DPSGD_ACT_GELU) {
      const float p = sigmoid(2.0f * kGelu0 * fmaf(kGelu1 * z[c] * z[c], z[c], z[c]));
      const float du = kGelu0 * fmaf(3.0f * kGelu1 * z[c], z[c], 1.0f);
      // Where p is 0 or 1 the first term is 0, also where du has left float32.
      const float w = 2.0f * z[c] * p * (1.0f - p);
      slope[c] = w == 0.0f ? p : fmaf(w, du, p);
    }
  }
}

// Rows of a thread's tile are worked on one after the other: interleaved, their
// intermediate values do not fit the registers beside the tile.
__device__ __forceinline__ void row_by_row() { __builtin_amdgcn_sched_barrier(0); }

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
  float* partials;       // forward: [B][chunks][blocks][segs][3]; backward: [B][chunks][C][2]
  float2* sums;          // [B][groups] m1, m2
  int32_t S, rows;       // rows of an example, of a tile
  int32_t B, C, groups, width;
  int32_t chunks, blocks;   // tiles of an example: row chunks, channel blocks
  int32_t units, segs;   // channel vectors of a block; most groups that a block has a part of
  int32_t by_xcd;        // order of the tiles (grid rounded up to whole rounds of examples)
  int32_t lanes, log;    // threads of a row, a power of two (log2: log) and at least units
  uint32_t magic;        // division by width
  int32_t shift;
  float eps;
};

// n values: their mean as an unevaluated sum hi + lo (lo at most a few roundings
// of hi), and the sum of squared deviations from it. The second word keeps the
// difference of two means, whose square enters the sum when they are merged, as
// exact as the values themselves when the mean is far larger than the spread.
struct Stat {
  float n, hi, lo, m2;
};

// Sum of squares about the mean of n values from that about a point which is
// `lo` below it; at least 0 (and NaN stays NaN).
__device__ __forceinline__ float about_mean(float m2, float n, float lo) {
  const float m = fmaf(-n * lo, lo, m2);
  return m < 0.0f ? 0.0f : m;
}

// An empty side is left alone: its mean of 0 says nothing, and the square of the
// other's distance from it may not be finite.
__device__ __forceinline__ void merge(Stat& a, const Stat& b) {
  if (b.n == 0.0f) return;
  if (a.n == 0.0f) {
    a = b;
    return;
  }
  const float t = a.n + b.n;
  const float w = b.n / t, d = (b.hi - a.hi) + (b.lo - a.lo);
  a.m2 = a.m2 + b.m2 + d * d * a.n * w;
  const float lo = fmaf(d, w, a.lo), hi = a.hi + lo;
  const float back = hi - a.hi;
  a.lo = (a.hi - (hi - back)) + (lo - back);
  a.hi = hi;
  a.n = t;
}

// Where a thread is: tile (example b, chunk, block), rows r0 + r + k step < r1,
// channels c .. c + V - 1 (in the block: unit V ...). first: first group of the
// block, of which it has a part.
struct Place {
  int32_t b, chunk, blk, r, r0, r1, step, unit, c, c0, c1, first, here;
  bool active;
};

template <int V>
__device__ __forceinline__ Place place_of(const GnArgs& a) {
  Place p;
  const uint32_t w = blockIdx.x, per = (uint32_t)a.blocks * (uint32_t)a.chunks;
  uint32_t rest;
  if (a.by_xcd) {   // workgroups go to the XCDs in turn: an example's tiles to one of them
    const uint32_t i = w / kXcds;
    p.b = (int32_t)(i / per * kXcds + w % kXcds);
    rest = i % per;
  } else {
    p.b = (int32_t)(w / per);
    rest = w - (uint32_t)p.b * per;
  }
  p.chunk = (int32_t)(rest / (uint32_t)a.blocks);
  p.blk = (int32_t)(rest - (uint32_t)p.chunk * (uint32_t)a.blocks);
  p.step = (int32_t)blockDim.x >> a.log;
  p.r = (int32_t)threadIdx.x >> a.log;
  p.unit = (int32_t)threadIdx.x & (a.lanes - 1);
  p.c0 = p.blk * a.units * V;
  p.c1 = p.c0 + a.units * V < a.C ? p.c0 + a.units * V : a.C;
  p.c = p.c0 + p.unit * V;
  p.active = p.unit < a.units && p.c < a.C;
  p.r0 = p.chunk * a.rows;
  p.r1 = a.S - p.r0 < a.rows ? a.S : p.r0 + a.rows;
  p.first = (int32_t)magic_divide((uint32_t)p.c0, a.magic, a.shift);
  p.here = (int32_t)magic_divide((uint32_t)p.c1 - 1, a.magic, a.shift) - p.first + 1;
  return p;
}

// Rows that a tile's sums are left in: one a wave where a wave has several rows
// of the block (those are added in registers), else one for each row of threads.
__host__ __device__ __forceinline__ int slots_of(int threads, int log) {
  return log < 6 ? threads >> 6 : threads >> log;
}

// A thread's V sums, added over the wave's rows, to lds[slot][channels].
template <int V>
__device__ __forceinline__ void leave_sums(float (&v)[V], const Place& p, const GnArgs& a,
                                           float* lds) {
  for (int off = 32; off >= a.lanes; off >>= 1) {
#pragma unroll
    for (int c = 0; c < V; ++c) v[c] += __shfl_xor(v[c], off, 64);
  }
  const int slot = a.log < 6 ? (int)threadIdx.x >> 6 : p.r;
  if (p.unit < a.units && (a.log >= 6 || (int)(threadIdx.x & 63) < a.lanes))
    store_vec<V>(lds + (slot * a.units + p.unit) * V, v);
}

// Channels of the block's j-th group that are in the block.
__device__ __forceinline__ int part_of(int j, const Place& p, const GnArgs& a) {
  const int g0 = (p.first + j) * a.width;
  return (g0 + a.width < p.c1 ? g0 + a.width : p.c1) - (g0 > p.c0 ? g0 : p.c0);
}

// The sum over the block's part of its j-th group, in every lane of a wave; lds
// holds `slots` values a channel.
__device__ __forceinline__ float group_sum(const float* lds, int slots, int channels, int j,
                                           const Place& p, const GnArgs& a) {
  const int lane = threadIdx.x & 63;
  const int g0 = (p.first + j) * a.width;
  const int from = (g0 > p.c0 ? g0 : p.c0) - p.c0;
  const int n = part_of(j, p, a);
  float s = 0.0f;
  if (n == a.width) {
    for (int k = lane; k < slots * n; k += 64) {
      const int i = (int)magic_divide((uint32_t)k, a.magic, a.shift);
      s += lds[i * channels + from + (k - i * n)];
    }
  } else {
    for (int i = 0; i < slots; ++i)
      for (int k = lane; k < n; k += 64) s += lds[i * channels + from + k];
  }
  return wave_total(s);
}

// Statistics of a tile; with WHOLE (all rows, whole groups) the output too.
template <class T, int V, int ACT, bool WHOLE>
__global__ __launch_bounds__(kTile, 8) void gn_tile_kernel(GnArgs a) {
  extern __shared__ __align__(16) float gn_lds[];
  const Place p = place_of<V>(a);
  if (p.b >= a.B) return;   // the whole workgroup
  const int channels = a.units * V, slots = slots_of(blockDim.x, a.log);
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  float* lds = gn_lds;                          // [2][slots][channels]
  float* seg_mean = lds + 2 * slots * channels; // [segs]
  float* seg_rstd = seg_mean + a.segs;          // [segs]
  const int64_t at = ((int64_t)p.b * a.S + p.r0 + p.r) * a.C + p.c, stride = (int64_t)p.step * a.C;
  const T* x = static_cast<const T*>(a.x) + at;
  const int32_t n_rows = p.r1 - p.r0;

  Raw<T, V> raw[kTileRows<T>];
  float v[V] = {};
#pragma unroll
  for (int k = 0; k < kTileRows<T>; ++k) {
    raw[k].zero();
    const int32_t r = p.r + k * p.step;
    if (p.active && r < n_rows) raw[k].load(x + k * stride);
  }
#pragma unroll
  for (int k = 0; k < kTileRows<T>; ++k) {
    float f[V];
    raw[k].widen(f);
#pragma unroll
    for (int c = 0; c < V; ++c) v[c] += f[c];
  }
  leave_sums<V>(v, p, a, lds);
  __syncthreads();
  for (int j = wave; j < p.here; j += waves) {
    const float s = group_sum(lds, slots, channels, j, p, a);
    if ((threadIdx.x & 63) == 0) seg_mean[j] = s / ((float)n_rows * (float)part_of(j, p, a));
  }
  __syncthreads();

  // The deviations from the mean of the tile's part of a group.
  float mu[V];
#pragma unroll
  for (int c = 0; c < V; ++c)
    mu[c] = p.active ? seg_mean[magic_divide((uint32_t)(p.c + c), a.magic, a.shift) - (uint32_t)p.first] : 0.0f;
  float q[V];
#pragma unroll
  for (int c = 0; c < V; ++c) v[c] = q[c] = 0.0f;
#pragma unroll
  for (int k = 0; k < kTileRows<T>; ++k) {
    if (p.r + k * p.step < n_rows) {
      float f[V];
      raw[k].keep_raw();
      raw[k].widen(f);
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float d = f[c] - mu[c];
        v[c] += d;
        q[c] = fmaf(d, d, q[c]);
      }
    }
  }
  if (!p.active) {
#pragma unroll
    for (int c = 0; c < V; ++c) v[c] = q[c] = 0.0f;
  }
  leave_sums<V>(v, p, a, lds);
  leave_sums<V>(q, p, a, lds + slots * channels);
  __syncthreads();
  for (int j = wave; j < p.here; j += waves) {
    const float s = group_sum(lds, slots, channels, j, p, a);
    const float t = group_sum(lds + slots * channels, slots, channels, j, p, a);
    if ((threadIdx.x & 63) == 0) {
      if constexpr (WHOLE) {
        // The group's mean and rstd, for everyone.
        const float count = (float)a.S * (float)a.width, lo = s / count;
        const float mean = seg_mean[j] + lo;
        const float rstd = 1.0f / sqrtf(about_mean(t, count, lo) / count + a.eps);
        const int64_t g = (int64_t)p.b * a.groups + p.first + j;
        a.mean[g] = seg_mean[j] = mean;
        a.rstd[g] = seg_rstd[j] = rstd;
      } else {
        const float count = (float)n_rows * (float)part_of(j, p, a), lo = s / count;
        float* to = a.partials + ((int64_t)blockIdx.x * a.segs + j) * 3;
        to[0] = seg_mean[j];
        to[1] = lo;
        to[2] = about_mean(t, count, lo);
      }
    }
  }

  if constexpr (WHOLE) {
    __syncthreads();
    // The thread's place once more, so that no register holds it until here.
    int32_t tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int32_t r = tid >> a.log, unit = tid & (a.lanes - 1), ch = p.c0 + unit * V;
    if (unit >= a.units || ch >= a.C) return;
    float ga[V], be[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int32_t s = (int32_t)magic_divide((uint32_t)(ch + c), a.magic, a.shift) - p.first;
      mu[c] = seg_mean[s];
      ga[c] = a.gamma ? seg_rstd[s] * a.gamma[ch + c] : seg_rstd[s];
      be[c] = a.beta ? a.beta[ch + c] : 0.0f;
    }
    T* y = static_cast<T*>(a.out) + ((int64_t)p.b * a.S + r) * a.C + ch;
#pragma unroll
    for (int k = 0; k < kTileRows<T>; ++k) {
      if (r + k * p.step < n_rows) {
        float f[V];
        raw[k].keep_raw();
        raw[k].widen(f);
#pragma unroll
        for (int c = 0; c < V; ++c) f[c] = fmaf(f[c] - mu[c], ga[c], be[c]);
        activate<ACT, V>(f);
        store_vec<V>(y + k * stride, f);
        row_by_row();
      }
    }
  }
}

// One workgroup per example and group: the tiles' statistics merged, each
// thread a range of them, then pairwise.
__global__ __launch_bounds__(kThreads) void gn_finish_kernel(GnArgs a) {
  __shared__ float lds[kThreads][4];
  const uint32_t b = blockIdx.x / (uint32_t)a.groups;
  const int32_t g = (int32_t)(blockIdx.x - b * (uint32_t)a.groups);
  // Blocks that have a part of the group (channels of a block: `per`).
  const int32_t per = a.units, g0 = g * a.width, g1 = g0 + a.width;
  const int32_t k0 = g0 / per, n_blocks = (g1 - 1) / per - k0 + 1;
  Stat st{};
  for (int32_t k = threadIdx.x; k < a.chunks * n_blocks; k += kThreads) {
    const int32_t chunk = k / n_blocks, blk = k0 + k - chunk * n_blocks;
    const int32_t c0 = blk * per, c1 = c0 + per < a.C ? c0 + per : a.C;
    const float* s = a.partials + ((((int64_t)b * a.chunks + chunk) * a.blocks + blk) * a.segs +
                                   (g - c0 / a.width)) * 3;
    const int32_t rows = a.S - chunk * a.rows < a.rows ? a.S - chunk * a.rows : a.rows;
    const int32_t n = (g1 < c1 ? g1 : c1) - (g0 > c0 ? g0 : c0);
    merge(st, Stat{(float)rows * (float)n, s[0], s[1], s[2]});
  }
  float* mine = lds[threadIdx.x];
  for (int half = kThreads / 2; half >= 1; half >>= 1) {
    mine[0] = st.n;
    mine[1] = st.hi;
    mine[2] = st.lo;
    mine[3] = st.m2;
    __syncthreads();
    if ((int)threadIdx.x < half) {
      const float* o = lds[threadIdx.x + half];
      merge(st, Stat{o[0], o[1], o[2], o[3]});
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    a.mean[blockIdx.x] = st.hi + st.lo;   // a statistic that was merged with nothing still has both
    a.rstd[blockIdx.x] = 1.0f / sqrtf(st.m2 / ((float)a.S * (float)a.width) + a.eps);
  }
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(kTile) void gn_apply_kernel(GnArgs a) {
  const Place p = place_of<V>(a);
  if (!p.active) return;
  const int64_t at = ((int64_t)p.b * a.S + p.r0) * a.C + p.c;
  const T* x = static_cast<const T*>(a.x) + at;
  T* y = static_cast<T*>(a.out) + at;
  float mu[V], rs[V], ga[V], be[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int64_t g = (int64_t)p.b * a.groups + magic_divide((uint32_t)(p.c + c), a.magic, a.shift);
    mu[c] = a.mean[g];
    rs[c] = a.rstd[g];
    ga[c] = a.gamma ? a.gamma[p.c + c] : 1.0f;
    be[c] = a.beta ? a.beta[p.c + c] : 0.0f;
  }
  const int32_t n_rows = p.r1 - p.r0;
#pragma unroll 4
  for (int32_t r = p.r; r < n_rows; r += p.step) {
    float v[V];
    load_vec<V>(x + (int64_t)r * a.C, v);
#pragma unroll
    for (int c = 0; c < V; ++c) v[c] = fmaf((v[c] - mu[c]) * rs[c], ga[c], be[c]);
    activate<ACT, V>(v);
    store_vec<V>(y + (int64_t)r * a.C, v);
  }
}

// Sums of a tile's dz and dz xh; with WHOLE dgamma_i, dbeta_i and dx too.
template <class T, int V, int ACT, bool WHOLE>
__global__ __launch_bounds__(kTile) void gn_grad_tile_kernel(GnArgs a) {
  extern __shared__ __align__(16) float gn_lds[];
  const Place p = place_of<V>(a);
  if (p.b >= a.B) return;   // the whole workgroup
  const int channels = a.units * V, slots = slots_of(blockDim.x, a.log);
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  float* lds = gn_lds;                          // [2][slots][channels]
  float* weighted = lds + 2 * slots * channels; // [2][channels]: gamma times a channel's sums
  float* seg = weighted + 2 * channels;         // [segs][2]
  const int64_t at = ((int64_t)p.b * a.S + p.r0 + p.r) * a.C + p.c, stride = (int64_t)p.step * a.C;
  const T* x = static_cast<const T*>(a.x) + at;
  const T* dy = static_cast<const T*>(a.dy) + at;
  const int32_t n_rows = p.r1 - p.r0;

  float rs[V], mu[V], ga[V], be[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    rs[c] = mu[c] = be[c] = 0.0f;
    ga[c] = 1.0f;
    if (p.active) {
      const int64_t g = (int64_t)p.b * a.groups + magic_divide((uint32_t)(p.c + c), a.magic, a.shift);
      rs[c] = a.rstd[g];
      mu[c] = a.mean[g];
      if (a.gamma) ga[c] = a.gamma[p.c + c];
      if (a.beta) be[c] = a.beta[p.c + c];
    }
  }
  Raw<T, V> rx[kGradRows], rd[kGradRows];
#pragma unroll
  for (int k = 0; k < kGradRows; ++k) {
    rx[k].zero();
    rd[k].zero();
    const int32_t r = p.r + k * p.step;
    if (p.active && r < n_rows) {
      rx[k].load(x + k * stride);
      rd[k].load(dy + k * stride);
    }
  }
  float sb[V] = {}, sg[V] = {};
  float dz[kGradRows][V];
#pragma unroll
  for (int k = 0; k < kGradRows; ++k) {
    float xv[V], z[V], slope[V];
    rx[k].widen(xv);
    rd[k].widen(dz[k]);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      xv[c] = (xv[c] - mu[c]) * rs[c];
      z[c] = fmaf(xv[c], ga[c], be[c]);
    }
    slopes<ACT, V>(z, slope);
    const bool there = p.active && p.r + k * p.step < n_rows;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      dz[k][c] = there ? dz[k][c] * slope[c] : 0.0f;
      sb[c] += dz[k][c];
      sg[c] += there ? dz[k][c] * xv[c] : 0.0f;
      if constexpr (sizeof(T) == 4 && WHOLE) rx[k].w[c] = __float_as_uint(xv[c]);   // xh in x's place
    }
    row_by_row();
  }
  leave_sums<V>(sb, p, a, lds);
  leave_sums<V>(sg, p, a, lds + slots * channels);
  __syncthreads();
  // One pair a channel, to its place in the tile's or the example's sums.
  for (int k = threadIdx.x; k < p.c1 - p.c0; k += blockDim.x) {
    float s = 0.0f, t = 0.0f;
#pragma unroll 4
    for (int i = 0; i < slots; ++i) {
      s += lds[i * channels + k];
      t += lds[(slots + i) * channels + k];
    }
    if constexpr (WHOLE) {
      a.dbeta[(int64_t)p.b * a.C + p.c0 + k] = s;
      a.dgamma[(int64_t)p.b * a.C + p.c0 + k] = t;
      const float w = a.gamma ? a.gamma[p.c0 + k] : 1.0f;
      weighted[k] = w * s;
      weighted[channels + k] = w * t;
    } else {
      reinterpret_cast<float2*>(a.partials)[((int64_t)p.b * a.chunks + p.chunk) * a.C + p.c0 + k] =
          make_float2(s, t);
    }
  }
  if constexpr (WHOLE) {
    __syncthreads();
    for (int j = wave; j < p.here; j += waves) {
      const float s = group_sum(weighted, 1, channels, j, p, a);
      const float t = group_sum(weighted + channels, 1, channels, j, p, a);
      if ((threadIdx.x & 63) == 0) {
        seg[2 * j] = s;
        seg[2 * j + 1] = t;
      }
    }
    __syncthreads();
    if (!p.active) return;
    const float inv = 1.0f / ((float)a.S * (float)a.width);
    float m1[V], m2[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const int32_t j = (int32_t)magic_divide((uint32_t)(p.c + c), a.magic, a.shift) - p.first;
      m1[c] = seg[2 * j] * inv;
      m2[c] = seg[2 * j + 1] * inv;
    }
    T* dx = static_cast<T*>(a.out) + at;
#pragma unroll
    for (int k = 0; k < kGradRows; ++k) {
      if (p.r + k * p.step < n_rows) {
        float xv[V];
        rx[k].keep_raw();
        rx[k].widen(xv);
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float xh = sizeof(T) == 4 ? xv[c] : (xv[c] - mu[c]) * rs[c];
          dz[k][c] = rs[c] * (fmaf(dz[k][c], ga[c], -m1[c]) - xh * m2[c]);
        }
        store_vec<V>(dx + k * stride, dz[k]);
        row_by_row();
      }
    }
  }
}

// One workgroup per example and group: dgamma_i and dbeta_i of its channels, and
// the means m1 and m2. Up to kThreads / width threads add a channel's tiles.
__global__ __launch_bounds__(kThreads) void gn_grad_finish_kernel(GnArgs a) {
  __shared__ float2 lds[kThreads];
  __shared__ float red[kThreads / 64];
  const uint32_t b = blockIdx.x / (uint32_t)a.groups;
  const int32_t g = (int32_t)(blockIdx.x - b * (uint32_t)a.groups);
  const int32_t wide = a.width < kThreads ? a.width : kThreads, h = kThreads / wide;
  const int32_t j = threadIdx.x / wide, k0 = threadIdx.x - j * wide;
  float s1 = 0.0f, s2 = 0.0f;
  for (int32_t base = 0; base < a.width; base += wide) {
    const int32_t k = base + k0;
    const int64_t c = (int64_t)g * a.width + k;
    float2 s = make_float2(0.0f, 0.0f);
    if (j < h && k < a.width) {
#pragma unroll 4
      for (int32_t chunk = j; chunk < a.chunks; chunk += h) {
        const float2 q = reinterpret_cast<const float2*>(a.partials)[((int64_t)b * a.chunks + chunk) * a.C + c];
        s.x += q.x;
        s.y += q.y;
      }
    }
    lds[threadIdx.x] = s;
    __syncthreads();
    if (j == 0 && k < a.width) {
      for (int32_t i = 1; i < h; ++i) {
        s.x += lds[i * wide + k0].x;
        s.y += lds[i * wide + k0].y;
      }
      a.dbeta[(int64_t)b * a.C + c] = s.x;
      a.dgamma[(int64_t)b * a.C + c] = s.y;
      const float ga = a.gamma ? a.gamma[c] : 1.0f;
      s1 = fmaf(ga, s.x, s1);
      s2 = fmaf(ga, s.y, s2);
    }
    __syncthreads();
  }
  s1 = block_sum(s1, red);
  s2 = block_sum(s2, red);
  const float inv = 1.0f / ((float)a.S * (float)a.width);
  if (threadIdx.x == 0) a.sums[blockIdx.x] = make_float2(s1 * inv, s2 * inv);
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(kTile) void gn_grad_apply_kernel(GnArgs a) {
  const Place p = place_of<V>(a);
  if (!p.active) return;
  const int64_t at = ((int64_t)p.b * a.S + p.r0) * a.C + p.c;
  const T* x = static_cast<const T*>(a.x) + at;
  const T* dy = static_cast<const T*>(a.dy) + at;
  T* dx = static_cast<T*>(a.out) + at;
  float mu[V], rs[V], ga[V], be[V], m1[V], m2[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const int64_t g = (int64_t)p.b * a.groups + magic_divide((uint32_t)(p.c + c), a.magic, a.shift);
    mu[c] = a.mean[g];
    rs[c] = a.rstd[g];
    ga[c] = a.gamma ? a.gamma[p.c + c] : 1.0f;
    be[c] = a.beta ? a.beta[p.c + c] : 0.0f;
    m1[c] = a.sums[g].x;
    m2[c] = a.sums[g].y;
  }
  const int32_t n_rows = p.r1 - p.r0;
#pragma unroll 4
  for (int32_t r = p.r; r < n_rows; r += p.step) {
    float v[V], d[V], z[V], slope[V];
    load_vec<V>(x + (int64_t)r * a.C, v);
    load_vec<V>(dy + (int64_t)r * a.C, d);
#pragma unroll
    for (int c = 0; c < V; ++c) {
      v[c] = (v[c] - mu[c]) * rs[c];
      z[c] = fmaf(v[c], ga[c], be[c]);
    }
    slopes<ACT, V>(z, slope);
#pragma unroll
    for (int c = 0; c < V; ++c) d[c] = rs[c] * (fmaf(d[c] * slope[c], ga[c], -m1[c]) - v[c] * m2[c]);
    store_vec<V>(dx + (int64_t)r * a.C, d);
  }
}

// Tiles of one direction: `per_thread` rows of a thread.
struct GnPlan {
  int vec, threads, units, lanes, log, blocks, segs;
  int64_t chunks, rows;
  bool whole, by_xcd;
};

// Channels of a block that are whole groups and whole vectors: the smallest
// number, then as many as make a row of the block `bytes` long.
int64_t block_channels(const dpsgd_group_norm& n, int vec, int64_t bytes) {
  const int64_t width = n.C / n.groups;
  int64_t least = width;
  while (least % vec != 0) least += width;   // at most vec steps
  int64_t cb = least * ceil_div(bytes, least * (n.dtype == DPSGD_BF16 ? 2 : 4));
  return cb < n.C ? cb : n.C;
}

// Threads of a row: the power of two from `units` on, so that rows lie in whole
// waves or waves in whole rows, and sums over a wave's rows are shuffles.
void set_lanes(GnPlan* p) {
  p->log = 0;
  while ((1 << p->log) < p->units) ++p->log;
  p->lanes = 1 << p->log;
}

GnPlan plan_of(const dpsgd_group_norm& n, int per_thread) {
  GnPlan p;
  p.vec = vec_width(n.C, 4);
  const int64_t width = n.C / n.groups;
  // All rows of a block of whole groups in one tile, where that fits: rows of 128
  // bytes, or else of 64, whose lines two tiles then share through one XCD's L2
  // ([256, 1024, 64] float32: 35 and 39 us forward and backward with 128 bytes, 47
  // and 59 with 64, 55 and 68 with 64 in plain order, 52 and 64 in three launches).
  for (int64_t bytes : {128, 64}) {
    const int64_t cb = block_channels(n, p.vec, bytes), units = ceil_div(cb, p.vec);
    if (units > kTile) continue;
    p.units = (int)units;
    set_lanes(&p);
    if (ceil_div(n.S, kTile / p.lanes) > per_thread) continue;
    p.whole = true;
    p.blocks = (int)ceil_div(n.C, cb);
    // As many threads as one row each takes, within a workgroup.
    const int64_t threads = round_up((size_t)(p.lanes * n.S), 64);
    p.threads = (int)(threads < kTile ? threads : kTile);
    p.chunks = 1;
    p.rows = n.S;
    p.segs = (int)(cb / width);
    p.by_xcd = bytes < 128 && p.blocks > 1 && n.B >= 64;
    return p;
  }
  p.whole = p.by_xcd = false;
  // Blocks of 128 bytes where rows are whole lines, so that no lane is idle at
  // C = 320, of 256 where neighbouring blocks share lines; wider for few rows.
  // [2, 16384, 320] bf16, forward and backward: 27 and 33 us, 29 and 40 with all
  // channels in tiles of 1024 threads ([4, 9000, 1030]: 82 and 101, 113 and 124;
  // [2, 16384, 324]: 29 and 40, 28 and 38, and 33 and 47 with blocks of 128 bytes).
  // Tiles of 512 threads take 29 and 35 us, of 128 threads 29 and 34.
  p.threads = kPartTile;
  const int64_t units = n.C / p.vec, elem = n.dtype == DPSGD_BF16 ? 2 : 4;
  int64_t most = (n.C * elem % 128 == 0 ? 128 : 256) / (p.vec * elem);
  while (most * n.S < kPartTile) most *= 2;
  p.units = (int)(units < most ? units : most);
  p.blocks = (int)ceil_div(units, p.units);
  set_lanes(&p);
  p.rows = (int64_t)per_thread * (kPartTile / p.lanes);
  if (p.rows > n.S) p.rows = n.S;
  p.chunks = ceil_div(n.S, p.rows);
  p.segs = (int)((int64_t)p.units * p.vec / width + 2);
  return p;
}

int rows_of(const dpsgd_group_norm& n, bool backward) {
  return backward ? kGradRows : n.dtype == DPSGD_BF16 ? kTileRows<uint16_t> : kTileRows<float>;
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
  a.S = (int32_t)n.S;
  a.rows = (int32_t)p.rows;
  a.B = (int32_t)n.B;
  a.C = (int32_t)n.C;
  a.groups = (int32_t)n.groups;
  a.width = (int32_t)(n.C / n.groups);
  a.chunks = (int32_t)p.chunks;
  a.blocks = p.blocks;
  a.units = p.units;
  a.segs = p.segs;
  a.by_xcd = p.by_xcd;
  a.lanes = p.lanes;
  a.log = p.log;
  divide_magic(n.C / n.groups, &a.magic, &a.shift);
  a.eps = n.eps;
  return a;
}

template <class T, int V, int ACT>
int run(const dpsgd_group_norm& n, const GnPlan& p, bool backward, GnArgs a, hipStream_t stream) {
  const int64_t B = p.by_xcd ? (int64_t)round_up((size_t)n.B, kXcds) : n.B;
  const int64_t tiles = B * p.chunks * p.blocks, groups = n.B * n.groups;
  // Launches that cannot be made are refused before the first.
  if (!launchable(tiles, p.threads) || (!p.whole && !launchable(groups, kThreads)))
    return DPSGD_ERR_INVALID_ARG;
  const dim3 grid((uint32_t)tiles), block((uint32_t)p.threads), by_group((uint32_t)groups);
  const size_t channels = (size_t)p.units * V, sums = 2 * (size_t)slots_of(p.threads, p.log) * channels;
  if (!backward) {
    const size_t lds = (sums + 2 * (size_t)p.segs) * sizeof(float);
    if (p.whole) {
      hipLaunchKernelGGL((gn_tile_kernel<T, V, ACT, true>), grid, block, lds, stream, a);
      return check_launch();
    }
    hipLaunchKernelGGL((gn_tile_kernel<T, V, DPSGD_ACT_NONE, false>), grid, block, lds, stream, a);
    GnArgs f = a;
    f.units = p.units * V;   // channels of a block
    hipLaunchKernelGGL(gn_finish_kernel, by_group, dim3(kThreads), 0, stream, f);
    hipLaunchKernelGGL((gn_apply_kernel<T, V, ACT>), grid, block, 0, stream, a);
    return check_launch();
  }
  const size_t lds = (sums + 2 * channels + 2 * (size_t)p.segs) * sizeof(float);
  if (p.whole) {
    hipLaunchKernelGGL((gn_grad_tile_kernel<T, V, ACT, true>), grid, block, lds, stream, a);
    return check_launch();
  }
  hipLaunchKernelGGL((gn_grad_tile_kernel<T, V, ACT, false>), grid, block, lds, stream, a);
  hipLaunchKernelGGL(gn_grad_finish_kernel, by_group, dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL((gn_grad_apply_kernel<T, V, ACT>), grid, block, 0, stream, a);
  return check_launch();
}

template <class T, int V>
int run_act(const dpsgd_group_norm& n, const GnPlan& p, bool backward, const GnArgs& a,
            hipStream_t stream) {
  switch (n.act) {
    case DPSGD_ACT_RELU: return run<T, V, DPSGD_ACT_RELU>(n, p, backward, a, stream);
    case DPSGD_ACT_SILU: return run<T, V, DPSGD_ACT_SILU>(n, p, backward, a, stream);
    case DPSGD_ACT_GELU: return run<T, V, DPSGD_ACT_GELU>(n, p, backward, a, stream);
    default: return run<T, V, DPSGD_ACT_NONE>(n, p, backward, a, stream);
  }
}

int run_group_norm(const dpsgd_group_norm& n, const GnPlan& p, bool backward, const GnArgs& a,
                   hipStream_t stream) {
  if (n.dtype == DPSGD_BF16) {
    switch (p.vec) {
      case 4: return run_act<uint16_t, 4>(n, p, backward, a, stream);
      case 2: return run_act<uint16_t, 2>(n, p, backward, a, stream);
      default: return run_act<uint16_t, 1>(n, p, backward, a, stream);
    }
  }
  switch (p.vec) {
    case 4: return run_act<float, 4>(n, p, backward, a, stream);
    case 2: return run_act<float, 2>(n, p, backward, a, stream);
    default: return run_act<float, 1>(n, p, backward, a, stream);
  }
}

}  // namespace

// Workspace: mean and rstd where the caller does not take them (backward: m1 and
// m2), then the tiles' statistics.
size_t group_norm_workspace_bytes(const dpsgd_group_norm& n) {
  const GnPlan f = plan_of(n, rows_of(n, false)), b = plan_of(n, rows_of(n, true));
  const size_t forward = f.whole ? 0 : (size_t)(n.B * f.chunks * f.blocks * f.segs) * 3 * sizeof(float);
  const size_t backward = b.whole ? 0 : (size_t)(n.B * b.chunks * n.C) * 2 * sizeof(float);
  return 2 * stat_bytes(n) + (forward > backward ? forward : backward);
}

int launch_group_norm_forward(const dpsgd_group_norm& n, const void* x, void* y, float* mean,
                              float* rstd, void* workspace, hipStream_t stream) {
  const GnPlan p = plan_of(n, rows_of(n, false));
  GnArgs a = args_of(n, p, x, y, workspace);
  if (mean) a.mean = mean;
  if (rstd) a.rstd = rstd;
  return run_group_norm(n, p, false, a, stream);
}

int launch_group_norm_backward(const dpsgd_group_norm& n, const void* x, const void* dy,
                               const float* mean, const float* rstd, void* dx, float* dgamma,
                               float* dbeta, void* workspace, hipStream_t stream) {
  const GnPlan p = plan_of(n, rows_of(n, true));
  GnArgs a = args_of(n, p, x, dx, workspace);
  a.dy = dy;
  a.mean = const_cast<float*>(mean);   // read only in the backward kernels
  a.rstd = const_cast<float*>(rstd);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  return run_group_norm(n, p, true, a, stream);
}

}  // namespace dpsgd
