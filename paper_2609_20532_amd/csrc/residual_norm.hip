// The residual sum between two blocks with the norms on both sides of it, and its
// gradients. Per row of C channels:
//
//   u = norm(block) post_gamma + post_beta;  r = alpha x + gate u;  y = norm(r) gamma + beta
//
//   D(g, vh) = rstd (g - mean(g) - vh mean(g vh))     (RMS: without mean(g))
//   dR = dr + D(dy gamma, rh);  dx = alpha dR;  dU = gate dR;  dblock = D(dU post_gamma, bh)
//   per example: dgamma = sum_s dy rh, dbeta = sum_s dy, dgate = sum_s dR u,
//                dpost_gamma = sum_s dU bh, dpost_beta = sum_s dU
//
// Bound by memory traffic: forward 4 rows of C elements (x, block, r, y), backward
// 6 (r, block, dy, dr, dx, dblock), each touched once. A group of threads has a row
// in registers, a fixed set of channels a thread, and takes several rows: up to 8192
// channels the affine parameters stay in registers, and so do the per-example sums of a
// backward group, which are joined over a workgroup's groups in LDS and over an example's workgroups
// by a second launch. Rows of whole waves have wave-uniform addresses.
//
// [16, 1024, 4096] in bf16, RMS norms on both sides and a gate: forward 103 us (537 MB,
// 5.2 TB/s), backward 169 us (806 MB and 25 MB of partial sums, 4.9 TB/s) and 5.5 for the
// join. [64, 128, 768], layer norm: backward 16.8 and 3.5 us (63 MB). A backward that has
// the next row's loads in flight while one is worked on needs 150 registers, so that a CU
// holds one workgroup of 512 threads in place of two (238 us in place of 169); for rows of
// fewer threads it was not tried. float32, [16, 1024, 4096]: forward 207 us (5.2 TB/s).
#include <math.h>

#include "vec.h"

namespace dpsgd {
namespace {

constexpr int kMostThreads = 1024;
constexpr int kWaves = kMostThreads / 64;
constexpr int kGrads = 5;   // dgamma, dbeta, dgate, dpost_gamma, dpost_beta

struct RnArgs {
  const void* x;         // backward: r
  const void* block;     // may be null
  const void* dy;
  const void* dr;        // may be null
  void* r;               // backward: dx (may be null)
  void* y;               // backward: dblock (null without a block)
  float* stats;          // [B S][4]
  const float* gamma;    // null: 1
  const float* beta;     // null: 0
  const float* post_gamma;
  const float* post_beta;
  const float* gate;
  float* grads[kGrads];  // [B][C], or null
  float* partials;       // [n_grads][B][chunks][C]
  int32_t n_grads;       // gradients that are asked for: which of them, and their places
  int32_t which[kGrads], place[kGrads];
  int64_t rows;          // B S
  int64_t S;
  int32_t C, log;        // log2 of the threads of a row
  int32_t iters;         // rows of a group
  int32_t chunks;        // backward: workgroups of an example
  int32_t gate_per_example, post, layer;
  float alpha, eps, inv_C;
  uint32_t magic;   // division by S
  int32_t shift;
};

// Elements of a thread. Forward: the work of a row that is the same for all of its
// threads is spread over more of them with 16 (16384 rows of 4096 in bf16: 105 us, 127
// with 8). Backward: 16 need 208 registers and spill in rows of 1024 threads (4096 rows
// of 8192, both by 512 workgroups: 110 us, 371 with 16; 175 us for 16384 rows of 4096
// either way).
constexpr int kForwardElements = 16, kBackwardElements = 8;

// Sums of K values over the threads of each row, in all of them. For rows of more
// than a wave every thread of the workgroup has to call it; `slot` goes between 0
// and 1 from call to call, so that one barrier a call is enough.
template <int K>
__device__ __forceinline__ void row_sum(float (&v)[K], int log, float (*lds)[kWaves][2], int& slot) {
  if (log < 6) {
    for (int off = 1; off < (1 << log); off <<= 1) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], off, 64);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_total(v[k]);
  if (log == 6) return;
  const int wave = threadIdx.x >> 6, per = 1 << (log - 6), from = wave & ~(per - 1);
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) lds[slot][wave][k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.0f;
  for (int w = 0; w < per; ++w) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += lds[slot][from + w][k];
  }
  slot ^= 1;
}

// A row's (or a parameter's) vectors of V elements that a thread has.
template <int V, int NV>
struct Channels {
  int32_t first, step, C;
  __device__ __forceinline__ int32_t at(int j) const { return first + j * step; }
  __device__ __forceinline__ bool has(int j) const { return at(j) < C; }
};

template <class T, int V, int NV>
__device__ __forceinline__ void load_row(const T* p, const Channels<V, NV>& ch, bool active,
                                         Raw<T, V> (&raw)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    raw[j].zero();
    if (active && ch.has(j)) raw[j].load(p + ch.at(j));
  }
}

template <class T, int V, int NV>
__device__ __forceinline__ void widen_row(const Raw<T, V> (&raw)[NV], float (&x)[NV][V]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) raw[j].widen(x[j]);
}

template <class T, int V, int NV>
__device__ __forceinline__ void store_row(T* p, const Channels<V, NV>& ch, const float (&x)[NV][V]) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (ch.has(j)) store_vec<V>(p + ch.at(j), x[j]);
}

template <int V, int NV>
__device__ __forceinline__ void load_affine(const float* p, float none, const Channels<V, NV>& ch,
                                            float (&x)[NV][V]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int c = 0; c < V; ++c) x[j][c] = none;
    if (p && ch.has(j)) load_vec<V>(p + ch.at(j), x[j]);
  }
}

// x rounded to the row's type and widened again.
template <class T, int V>
__device__ __forceinline__ void round_to(float (&x)[V]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int c = 0; c < V; ++c) x[c] = bf16_lo(pack_bf16x2(x[c], 0.0f));
  }
}

// 1 / sqrt(x): the hardware's, and a step of Newton's iteration, which needs x far from
// both ends of float32.
__device__ __forceinline__ float inverse_root(float x) {
  if (!(x > 0x1p-100f && x < 0x1p100f)) return 1.0f / sqrtf(x);
  const float y = __builtin_amdgcn_rsqf(x), e = fmaf(-x * y, y, 1.0f);
  return fmaf(0.5f * y, e, y);
}

// Mean (0 without `layer`) and rstd of a row in registers, channels past the end 0.
template <int V, int NV>
__device__ __forceinline__ float2 row_stats(const float (&x)[NV][V], const Channels<V, NV>& ch,
                                            const RnArgs& a, float (*lds)[kWaves][2], int& slot) {
  float s[1] = {0.0f}, mean = 0.0f;
  if (a.layer) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) s[0] += x[j][c];
    row_sum<1>(s, a.log, lds, slot);
    mean = s[0] * a.inv_C;
    s[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float t = 0.0f;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float d = x[j][c] - mean;
        t = fmaf(d, d, t);
      }
      s[0] += ch.has(j) ? t : 0.0f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) s[0] = fmaf(x[j][c], x[j][c], s[0]);
  }
  row_sum<1>(s, a.log, lds, slot);
  return make_float2(mean, inverse_root(fmaf(s[0], a.inv_C, a.eps)));
}

// Which of the workgroup's rows a thread has. WIDE: a row has whole waves, so that its
// addresses are the same for a wave (and are kept in scalar registers).
template <bool WIDE>
__device__ __forceinline__ int group_of(int log) {
  const int g = (int)threadIdx.x >> log;
  return WIDE ? __builtin_amdgcn_readfirstlane(g) : g;
}

// The five parameter arrays and two rows are in registers also above 8192 channels, where
// they spill: vectors of 4 elements 2 (bf16) and 14, of 2 39 and 46, of 1 154 (4 x 1024 rows of
// 12288 in float32: 203 us, 4.0 TB/s).
template <class T, int V, int NV, int MOST, bool WIDE>
__global__ __launch_bounds__(MOST) void rn_forward_kernel(RnArgs a) {
  __shared__ float lds[2][kWaves][2];
  const int group = group_of<WIDE>(a.log), groups = (int)blockDim.x >> a.log;
  const int lane = (int)threadIdx.x & ((1 << a.log) - 1);
  const Channels<V, NV> ch{lane * V, V << a.log, a.C};
  int slot = 0;
  float ga[NV][V], be[NV][V], gt[NV][V], pg[NV][V], pb[NV][V];
  load_affine<V, NV>(a.gamma, 1.0f, ch, ga);
  load_affine<V, NV>(a.beta, 0.0f, ch, be);
  load_affine<V, NV>(a.post_gamma, 1.0f, ch, pg);
  load_affine<V, NV>(a.post_beta, 0.0f, ch, pb);
  load_affine<V, NV>(a.gate_per_example ? nullptr : a.gate, 1.0f, ch, gt);
  uint32_t example = 0xFFFFFFFFu;   // whose gate this is
  for (int i = 0; i < a.iters; ++i) {
    const uint32_t row = (blockIdx.x * (uint32_t)a.iters + (uint32_t)i) * (uint32_t)groups + (uint32_t)group;
    const bool active = row < (uint32_t)a.rows;
    const int64_t at = (int64_t)row * a.C;
    Raw<T, V> rx[NV], rb[NV];
    load_row<T, V, NV>(static_cast<const T*>(a.x) + at, ch, active, rx);
    load_row<T, V, NV>(static_cast<const T*>(a.block) + at, ch, active && a.block, rb);
    if (a.gate_per_example && active) {
      const uint32_t e = magic_divide(row, a.magic, a.shift);
      if (e != example) load_affine<V, NV>(a.gate + (int64_t)e * a.C, 1.0f, ch, gt);
      example = e;
    }
    float x[NV][V], u[NV][V];
    widen_row<T, V, NV>(rx, x);
    widen_row<T, V, NV>(rb, u);
    float2 post = make_float2(0.0f, 0.0f);
    if (a.post) {
      post = row_stats<V, NV>(u, ch, a, lds, slot);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int c = 0; c < V; ++c) u[j][c] = fmaf((u[j][c] - post.x) * post.y, pg[j][c], pb[j][c]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int c = 0; c < V; ++c) x[j][c] = fmaf(gt[j][c], u[j][c], a.alpha * x[j][c]);
      if (!ch.has(j)) {
#pragma unroll
        for (int c = 0; c < V; ++c) x[j][c] = 0.0f;
      }
      round_to<T, V>(x[j]);
    }
    const float2 st = row_stats<V, NV>(x, ch, a, lds, slot);
    if (!active) continue;
    if (a.r) store_row<T, V, NV>(static_cast<T*>(a.r) + at, ch, x);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) x[j][c] = fmaf((x[j][c] - st.x) * st.y, ga[j][c], be[j][c]);
    store_row<T, V, NV>(static_cast<T*>(a.y) + at, ch, x);
    if (a.stats && lane == 0)
      reinterpret_cast<float4*>(a.stats)[row] = make_float4(st.x, st.y, post.x, post.y);
  }
}

// What a backward call needs: BARE no block's values (no norm of it, no gate's gradient),
// GATED the block as it is, POST the normed block.
enum BackKind : int { BARE = 0, GATED = 1, POST = 2 };

// One workgroup: some rows of one example, which its groups take in turn. The block's
// side has two sums, sum dR v (v: the normed block, or the block) and sum dR: gate and
// post_gamma are constant over an example, so dgate, dpost_gamma and dpost_beta are
// these times constants.
// Rows of more than 8 elements a thread (8193 to 16384 channels, 1024 threads, 128 registers
// each) are LEAN: gamma, gate and post_gamma are read again for each row (from L2), dr and the
// block when it is their turn, and the sums of dy rh and dy are in LDS, where a thread has its
// own places. In registers they spill 36 to 257 of them: 2 x 1024 rows of 16384 in bf16 85 us
// (116 with spills; with only the parameters read again 90), normed on both sides 127 (311;
// 269), 3 x 128 of 13502 with a gate 38 (74; 78). What still
// spills above 8192 channels: a norm of the block (vectors of 8, 4, 2 and 1 elements: 6, 23 to
// 27, 81 to 99 and 164 to 185 registers), a gate (vectors of 2 and 1: 21 to 23 and 66), neither
// (1 to 2 and 53 to 57), and one register in odd widths of 4097 to 8192 with a norm of the block.
template <class T, int V, int NV, int MOST, int KIND, bool WIDE>
__global__ __launch_bounds__(MOST) void rn_backward_kernel(RnArgs a) {
  extern __shared__ __align__(16) float rn_lds[];   // [groups][C], where there are several groups
  __shared__ float lds[2][kWaves][2];
  const int group = group_of<WIDE>(a.log), groups = (int)blockDim.x >> a.log;
  const int lane = (int)threadIdx.x & ((1 << a.log) - 1);
  const Channels<V, NV> ch{lane * V, V << a.log, a.C};
  const int64_t example = blockIdx.x / (uint32_t)a.chunks;
  const int32_t chunk = (int32_t)(blockIdx.x - (uint32_t)example * (uint32_t)a.chunks);
  const float* gate = a.gate ? a.gate + (a.gate_per_example ? example * a.C : 0) : nullptr;
  int slot = 0;
  constexpr bool LEAN = MOST == kMostThreads && NV * V > kBackwardElements;
  static_assert(!LEAN || NV * V == 16, "places of the sums");
  __shared__ float sums[LEAN ? 2 : 1][LEAN ? 16 * kMostThreads : 1];   // dy rh, dy
  const auto place = [&](int j, int c) { return (j * V + c) * kMostThreads + (int)threadIdx.x; };
  float ga[NV][V], gp[NV][V];   // gamma; gate post_gamma
  const auto load_gp = [&] {
    load_affine<V, NV>(gate, 1.0f, ch, gp);
    if constexpr (KIND == POST) {
      float pg[NV][V];
      load_affine<V, NV>(a.post_gamma, 1.0f, ch, pg);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int c = 0; c < V; ++c) gp[j][c] *= pg[j][c];
    }
  };
  if constexpr (LEAN) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) sums[0][place(j, c)] = sums[1][place(j, c)] = 0.0f;
  } else {
    load_affine<V, NV>(a.gamma, 1.0f, ch, ga);
    load_gp();
  }
  constexpr int kSums = KIND == POST ? 4 : (KIND == GATED ? 3 : 2);
  float acc[kSums][NV][V] = {};   // dy rh, dy, dR v, dR
  for (int i = 0; i < a.iters; ++i) {
    const int64_t s = ((int64_t)chunk * a.iters + i) * groups + group;
    const bool active = s < a.S;
    const int64_t row = example * a.S + s, at = row * a.C;
    Raw<T, V> rr[NV], rb[NV], rdy[NV], rdr[NV];
    load_row<T, V, NV>(static_cast<const T*>(a.x) + at, ch, active, rr);
    load_row<T, V, NV>(static_cast<const T*>(a.dy) + at, ch, active, rdy);
    const auto load_dr = [&] {
      load_row<T, V, NV>(static_cast<const T*>(a.dr) + at, ch, active && a.dr, rdr);
    };
    const auto load_block = [&] {
      if constexpr (KIND != BARE) load_row<T, V, NV>(static_cast<const T*>(a.block) + at, ch, active, rb);
    };
    if constexpr (!LEAN) load_dr(), load_block();
    float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (active) st = reinterpret_cast<const float4*>(a.stats)[row];
    float d[NV][V], vh[NV][V];
    widen_row<T, V, NV>(rdy, d);
    widen_row<T, V, NV>(rr, vh);
    float m[2] = {0.0f, 0.0f};
    if constexpr (LEAN) load_affine<V, NV>(a.gamma, 1.0f, ch, ga);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        vh[j][c] = ch.has(j) ? (vh[j][c] - st.x) * st.y : 0.0f;
        float& dg = LEAN ? sums[0][LEAN ? place(j, c) : 0] : acc[0][j][c];
        float& db = LEAN ? sums[1][LEAN ? place(j, c) : 0] : acc[1][j][c];
        dg = fmaf(d[j][c], vh[j][c], dg);
        db += d[j][c];
        d[j][c] *= ga[j][c];
        m[0] += d[j][c];
        m[1] = fmaf(d[j][c], vh[j][c], m[1]);
      }
    row_sum<2>(m, a.log, lds, slot);
    m[0] = a.layer ? m[0] * a.inv_C : 0.0f;
    m[1] *= a.inv_C;
    if constexpr (LEAN) load_dr();
    float dr[NV][V];
    widen_row<T, V, NV>(rdr, dr);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int c = 0; c < V; ++c) {
        dr[j][c] = fmaf(st.y, d[j][c] - fmaf(vh[j][c], m[1], m[0]), dr[j][c]);
        if (!ch.has(j)) dr[j][c] = 0.0f;
        d[j][c] = a.alpha * dr[j][c];
      }
    }
    if (active && a.r) store_row<T, V, NV>(static_cast<T*>(a.r) + at, ch, d);
    if (!a.y) continue;
    if constexpr (LEAN) load_gp(), load_block();
    if constexpr (KIND != BARE) widen_row<T, V, NV>(rb, vh);
    m[0] = m[1] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        d[j][c] = gp[j][c] * dr[j][c];
        if constexpr (KIND == POST) {
          vh[j][c] = ch.has(j) ? (vh[j][c] - st.z) * st.w : 0.0f;
          acc[3][j][c] += dr[j][c];
          m[0] += d[j][c];
          m[1] = fmaf(d[j][c], vh[j][c], m[1]);
        }
        if constexpr (KIND != BARE) acc[2][j][c] = fmaf(dr[j][c], vh[j][c], acc[2][j][c]);
      }
    if constexpr (KIND == POST) {
      row_sum<2>(m, a.log, lds, slot);
      m[0] = a.layer ? m[0] * a.inv_C : 0.0f;
      m[1] *= a.inv_C;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int c = 0; c < V; ++c) d[j][c] = st.w * (d[j][c] - fmaf(vh[j][c], m[1], m[0]));
    }
    if (active) store_row<T, V, NV>(static_cast<T*>(a.y) + at, ch, d);
  }

  // The groups' sums, added in their order, to the example's row or to a partial one.
#pragma unroll
  for (int k = 0; k < kGrads; ++k) {
    if (!a.grads[k]) continue;
    if (k >= (KIND == BARE ? 2 : (KIND == GATED ? 3 : kGrads))) continue;
    float* to = a.chunks == 1 ? a.grads[k] + example * a.C
                              : a.partials + ((int64_t)a.place[k] * gridDim.x + blockIdx.x) * a.C;
    float v[NV][V], f[NV][V];
    if (k >= 3) load_affine<V, NV>(gate, 1.0f, ch, f);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float pg[V], pb[V];
#pragma unroll
      for (int c = 0; c < V; ++c) pg[c] = 1.0f, pb[c] = 0.0f;
      if (KIND == POST && k == 2 && ch.has(j)) {
        if (a.post_gamma) load_vec<V>(a.post_gamma + ch.at(j), pg);
        if (a.post_beta) load_vec<V>(a.post_beta + ch.at(j), pb);
      }
#pragma unroll
      for (int c = 0; c < V; ++c) {
        if constexpr (KIND == POST)
          v[j][c] = k < 2 ? acc[k < 2 ? k : 0][j][c]
                          : (k == 2 ? fmaf(pb[c], acc[3][j][c], pg[c] * acc[2][j][c])
                                    : f[j][c] * acc[k == 3 ? 2 : 3][j][c]);
        else
          v[j][c] = acc[k < kSums ? k : 0][j][c];
        if constexpr (LEAN)
          if (k < 2) v[j][c] = sums[k][place(j, c)];
      }
    }
    if (groups == 1) {
      store_row<float, V, NV>(to, ch, v);
      continue;
    }
    __syncthreads();
    store_row<float, V, NV>(rn_lds + group * a.C, ch, v);
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
      float t = 0.0f;
      for (int g = 0; g < groups; ++g) t += rn_lds[g * a.C + c];
      to[c] = t;
    }
  }
}

// The workgroups' sums of an example, 64 channels a workgroup: four threads a channel
// add every fourth of them, in a fixed order.
__global__ __launch_bounds__(kThreads) void rn_join_kernel(RnArgs a, int32_t blocks, int64_t wgs) {
  __shared__ float part[4][64];
  const int32_t c0 = (int32_t)(blockIdx.x % (uint32_t)blocks) * 64, c = c0 + ((int32_t)threadIdx.x & 63);
  const uint32_t rest = blockIdx.x / (uint32_t)blocks;
  const int32_t n = a.n_grads, k = (int32_t)(rest % (uint32_t)n), way = (int32_t)threadIdx.x >> 6;
  const int64_t example = rest / (uint32_t)n;
  float t = 0.0f;
  if (c < a.C) {
    const float* from = a.partials + ((int64_t)k * wgs + example * a.chunks) * a.C + c;
#pragma unroll 8
    for (int32_t i = way; i < a.chunks; i += 4) t += from[(int64_t)i * a.C];
  }
  part[way][threadIdx.x & 63] = t;
  __syncthreads();
  if (way == 0 && c < a.C) {
    float* to = a.grads[a.which[k]];
    to[example * a.C + c] = (part[0][threadIdx.x] + part[1][threadIdx.x]) +
                            (part[2][threadIdx.x] + part[3][threadIdx.x]);
  }
}

// How a call is laid out: V elements a vector, nv vectors a thread, 2^log threads a
// row, `threads` a workgroup.
struct RnPlan {
  int V, nv, log, threads, groups;
  int iters;
  int64_t wgs, chunks;
};

// Vectors of V elements that a thread has of rows from a wave to 1024 threads. Fewer are for
// rows of at most a wave (256 threads a workgroup), more for those of 1024 threads.
constexpr int usual_vectors(int elements, int V) { return elements / V > 4 ? 4 : elements / V; }

RnPlan plan_rows(const dpsgd_residual_norm& n, int elements) {
  RnPlan p{};
  p.V = vec_width(n.C, n.dtype == DPSGD_BF16 ? 8 : 4);
  const int64_t units = n.C / p.V;
  p.nv = usual_vectors(elements, p.V);
  while (p.nv > 1 && units <= 64 * (p.nv / 2)) p.nv /= 2;
  while (units > (int64_t)p.nv * kMostThreads) p.nv *= 2;
  while (((int64_t)p.nv << p.log) < units) ++p.log;
  p.threads = p.log <= 8 ? kThreads : 1 << p.log;
  p.groups = p.threads >> p.log;
  return p;
}

// Workgroups that a call is spread over. Backward: each leaves its sums, which are read
// once more (the same rows of 4096: 175 us with 512, 196 with 1024, 200 with 256).
constexpr int64_t kForwardWgs = 4096, kBackwardWgs = 512;
// Of 1024 threads a CU holds one (2 x 1024 rows of 16384, before their sums were in LDS:
// 115 us with 256, 132 with 512).
constexpr int64_t kBackwardWideWgs = 256;
// A workgroup's sums are twice a row of bf16 for each gradient: where examples have few
// rows, each takes at least two batches while this many workgroups are left (8 x 64 rows of
// 4096: 17.5 us, one batch 20.9, four 18.6; 3 x 128 of 13502, likewise: 74 us, four batches 90).
constexpr int64_t kBackwardFewWgs = 128;

RnPlan plan_forward(const dpsgd_residual_norm& n) {
  RnPlan p = plan_rows(n, kForwardElements);
  const int64_t batches = ceil_div(n.B * n.S, p.groups);
  p.iters = (int)ceil_div(batches, kForwardWgs);
  p.wgs = ceil_div(batches, p.iters);
  return p;
}

RnPlan plan_backward(const dpsgd_residual_norm& n) {
  RnPlan p = plan_rows(n, kBackwardElements);
  while (p.threads > 64 && p.groups > 1 && p.groups / 2 >= n.S) {   // few rows: smaller workgroups
    p.threads /= 2;
    p.groups /= 2;
  }
  const int64_t batches = ceil_div(n.S, p.groups);
  const int64_t most = ceil_div(p.threads > 512 ? kBackwardWideWgs : kBackwardWgs, n.B);
  const int64_t few = ceil_div(kBackwardFewWgs, n.B), pairs = ceil_div(batches, 2);
  const int64_t enough = pairs > few ? pairs : few;
  const int64_t chunks = most < enough ? most : enough;
  p.iters = (int)ceil_div(batches, chunks < batches ? chunks : batches);
  p.chunks = ceil_div(batches, p.iters);
  p.wgs = n.B * p.chunks;
  return p;
}

RnArgs common_args(const dpsgd_residual_norm& n, const RnPlan& p) {
  RnArgs a{};
  a.gamma = n.gamma;
  a.beta = n.beta;
  a.post_gamma = n.post_gamma;
  a.post_beta = n.post_beta;
  a.gate = n.gate;
  a.rows = n.B * n.S;
  a.S = n.S;
  a.C = (int32_t)n.C;
  a.log = p.log;
  a.iters = p.iters;
  a.chunks = (int32_t)p.chunks;
  a.gate_per_example = n.gate && n.gate_per_example;
  a.post = n.post ? 1 : 0;
  a.layer = n.kind == DPSGD_ROW_NORM_LAYER;
  a.alpha = n.residual_scale;
  a.eps = n.eps;
  a.inv_C = 1.0f / (float)n.C;
  divide_magic(n.S, &a.magic, &a.shift);
  return a;
}

// FORWARD or a BackKind.
constexpr int FORWARD = -1;

template <class T, int V, int NV, int MOST, bool WIDE, int KIND>
int run(const RnPlan& p, const RnArgs& a, size_t lds, hipStream_t stream) {
  const dim3 grid((uint32_t)p.wgs), block(p.threads);
  if constexpr (KIND == FORWARD)
    hipLaunchKernelGGL((rn_forward_kernel<T, V, NV, MOST, WIDE>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((rn_backward_kernel<T, V, NV, MOST, KIND, WIDE>), grid, block, lds, stream, a);
  return check_launch();
}

// The kernels that a plan can ask for, and no others.
template <class T, int V, int NV, int KIND>
int pick_threads(const RnPlan& p, const RnArgs& a, size_t lds, hipStream_t stream) {
  constexpr int kUsual = usual_vectors(KIND == FORWARD ? kForwardElements : kBackwardElements, V);
  if constexpr (NV >= kUsual)
    if (p.threads > 512) return run<T, V, NV, kMostThreads, true, KIND>(p, a, lds, stream);
  if constexpr (NV == kUsual)
    if (p.threads > kThreads && p.threads <= 512) return run<T, V, NV, 512, true, KIND>(p, a, lds, stream);
  if constexpr (NV == 1)   // rows of less than a wave have one vector a thread
    if (p.log < 6) return run<T, V, NV, kThreads, false, KIND>(p, a, lds, stream);
  if constexpr (NV <= kUsual)
    if (p.threads <= kThreads) return run<T, V, NV, kThreads, true, KIND>(p, a, lds, stream);
  return DPSGD_ERR_UNSUPPORTED;
}

template <class T, int V, int KIND>
int pick_vectors(const RnPlan& p, const RnArgs& a, size_t lds, hipStream_t stream) {
  switch (p.nv) {
    case 1: return pick_threads<T, V, 1, KIND>(p, a, lds, stream);
    case 2: return pick_threads<T, V, 2, KIND>(p, a, lds, stream);
    case 4:
      if constexpr (V <= 4) return pick_threads<T, V, 4, KIND>(p, a, lds, stream);
      break;
    case 8:
      if constexpr (V <= 2) return pick_threads<T, V, 8, KIND>(p, a, lds, stream);
      break;
    case 16:
      if constexpr (V <= 1) return pick_threads<T, V, 16, KIND>(p, a, lds, stream);
      break;
  }
  return DPSGD_ERR_UNSUPPORTED;
}

template <int KIND>
int launch(const dpsgd_residual_norm& n, const RnPlan& p, const RnArgs& a, size_t lds,
           hipStream_t stream) {
  if (!launchable(p.wgs, p.threads)) return DPSGD_ERR_INVALID_ARG;
  if (n.dtype == DPSGD_BF16) {
    switch (p.V) {
      case 8: return pick_vectors<uint16_t, 8, KIND>(p, a, lds, stream);
      case 4: return pick_vectors<uint16_t, 4, KIND>(p, a, lds, stream);
      case 2: return pick_vectors<uint16_t, 2, KIND>(p, a, lds, stream);
      default: return pick_vectors<uint16_t, 1, KIND>(p, a, lds, stream);
    }
  }
  switch (p.V) {
    case 4: return pick_vectors<float, 4, KIND>(p, a, lds, stream);
    case 2: return pick_vectors<float, 2, KIND>(p, a, lds, stream);
    default: return pick_vectors<float, 1, KIND>(p, a, lds, stream);
  }
}

}  // namespace

size_t residual_norm_workspace_bytes(const dpsgd_residual_norm& n) {
  const RnPlan p = plan_backward(n);
  const size_t bytes = p.chunks == 1 ? 0 : (size_t)p.wgs * kGrads * (size_t)n.C * sizeof(float);
  return bytes + 16;
}

int launch_residual_norm_forward(const dpsgd_residual_norm& n, const void* x, const void* block,
                                 void* r, void* y, float* stats, hipStream_t stream) {
  const RnPlan p = plan_forward(n);
  RnArgs a = common_args(n, p);
  a.x = x;
  a.block = block;
  a.r = r;
  a.y = y;
  a.stats = stats;
  return launch<FORWARD>(n, p, a, 0, stream);
}

int launch_residual_norm_backward(const dpsgd_residual_norm& n, const void* block, const void* r,
                                  const void* dy, const void* dr, const float* stats, void* dx,
                                  void* dblock, float* const* grads, void* workspace,
                                  hipStream_t stream) {
  const RnPlan p = plan_backward(n);
  RnArgs a = common_args(n, p);
  a.x = r;
  a.block = block;
  a.dy = dy;
  a.dr = dr;
  a.stats = const_cast<float*>(stats);
  a.r = dx;
  a.y = dblock;
  a.partials = static_cast<float*>(workspace);
  for (int k = 0; k < kGrads; ++k) {
    a.grads[k] = grads[k];
    if (!grads[k]) continue;
    a.place[k] = a.n_grads;
    a.which[a.n_grads++] = k;
  }
  const size_t lds = a.n_grads && p.groups > 1 ? (size_t)p.groups * (size_t)n.C * sizeof(float) : 0;
  const int st = n.post ? launch<POST>(n, p, a, lds, stream)
                 : grads[2] ? launch<GATED>(n, p, a, lds, stream)
                                : launch<BARE>(n, p, a, lds, stream);
  if (st != DPSGD_OK || !a.n_grads || p.chunks == 1) return st;
  const int64_t blocks = ceil_div(n.C, 64), wgs = n.B * a.n_grads * blocks;
  if (!launchable(wgs, kThreads)) return DPSGD_ERR_INVALID_ARG;
  hipLaunchKernelGGL(rn_join_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, a, (int32_t)blocks, p.wgs);
  return check_launch();
}

}  // namespace dpsgd
