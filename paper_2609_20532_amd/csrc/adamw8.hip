// Noise + AdamW step whose moments are held in 8 bits.
//
//   g = scale (S + sigma C z);  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - lr_t m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory traffic: 16 bytes an entry (gradient and parameter read 4 each,
// parameter written 4, two codes read and written) in place of 28 with float32
// moments. A wave takes blocks of 256 entries, four neighbouring ones a lane, so
// that a block's exponents are maxima over one wave and nothing is shared between
// waves.
//
// 52.7 million entries with stochastic rounding: 153 us (846 MB, 5.5 TB/s; the moments in
// float32 would be 1.48 GB), read back in bf16 51-59 us (316 MB). A Philox block for four
// entries' random bits is about a quarter of the time that the arithmetic units have. 20
// matrices of 123 thousand entries together: 5.2 and 4.0 us.
//
// Codes are the upper bits of a float32: a magnitude scaled by a power of two so
// that its block's exponent becomes 15 (m) or 31 (v) has its code in bits 20 and
// up, with float32's subnormal numbers as the code's. Rounding is an integer
// addition below bit 20 and never carries past the highest code, because the
// block's exponent is that of the largest magnitude rounded up to 3 bits.
//
// Every operation is rounded by itself: the step is defined bit for bit, whatever
// a compiler would contract.
#include <math.h>

#include "philox.h"
#include "vec.h"

#pragma clang fp contract(off)

namespace dpsgd {
namespace {

constexpr int kStateBlock = DPSGD_STATE_BLOCK;
static_assert(kStateBlock == 4 * 64, "a wave takes a block, four entries a lane");
// Blocks of a wave, whose loads are in flight together: 4, or 1 where the tensors of a
// launch are small and its time is that of one wave (kFewBlocks: 8 waves a CU).
constexpr int kManyBlocks = 4;
constexpr int64_t kFewBlocks = 2048;
constexpr int blocks_per_wg(int per_wave) { return per_wave * kThreads / 64; }
constexpr int kTopM = 15, kTopV = 31;      // code exponents that stand for the block's
constexpr uint32_t kLowM = 32, kLowV = 48; // lowest block exponents
constexpr uint32_t kNotFinite = 255;

// Largest value of the wave in every lane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, off, 64);
    v = o > v ? o : v;
  }
  return v;
}

// A block's exponent from the largest bits of its magnitudes.
__device__ __forceinline__ uint32_t block_exponent(uint32_t bits, uint32_t lowest) {
  const uint32_t k = (bits + 0xFFFFFu) >> 23;
  return k < lowest ? lowest : (k > kNotFinite ? kNotFinite : k);
}

// The magnitude of a code (without the sign): exact.
__device__ __forceinline__ float code_value(uint32_t code, uint32_t k, int top) {
  const float x = ldexpf(__uint_as_float(code << 20), (int)k - top);
  return k == kNotFinite ? __uint_as_float(0x7FC00000u) : x;
}

__device__ __forceinline__ float value_m(uint32_t code, uint32_t k) {
  const float x = code_value(code & 127u, k, kTopM);
  return code & 128u ? -x : x;
}

__device__ __forceinline__ float value_v(uint32_t code, uint32_t k) {
  return code_value(code, k, kTopV);
}

// Code of a magnitude; r16: random bits of stochastic rounding.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t code_of(float x, uint32_t k, int top, uint32_t r16) {
  const uint32_t u = __float_as_uint(ldexpf(x, top - (int)k));
  if constexpr (STOCHASTIC) return (u + (r16 << 4)) >> 20;
  return (u + 0x7FFFFu + ((u >> 20) & 1u)) >> 20;
}

// Codes of four entries of a block, in the bytes of a word; 0 in a block that is
// not finite.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t codes_m(const float (&m)[4], uint32_t k, const uint32_t (&r)[4]) {
  uint32_t w = 0;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    w |= (code_of<STOCHASTIC>(fabsf(m[c]), k, kTopM, r[c] & 0xFFFFu) | (m[c] < 0.0f ? 128u : 0u))
         << (8 * c);
  return k == kNotFinite ? 0u : w;
}

template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t codes_v(const float (&v)[4], uint32_t k, const uint32_t (&r)[4]) {
  uint32_t w = 0;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t q = code_of<STOCHASTIC>(fabsf(v[c]), k, kTopV, r[c] >> 16);
    w |= (q == 0u && v[c] > 0.0f ? 1u : q) << (8 * c);
  }
  return k == kNotFinite ? 0u : w;
}

struct Seg8 {
  const float* grad;     // pack: m; unpack: not used
  float* param;          // pack: v (read only)
  uint8_t* m;
  uint8_t* v;
  uint8_t* exps;         // [blocks][2]
  float* noisy;          // may be null
  int64_t numel;
  uint32_t tensor_id;
  uint32_t wg_begin;
};

struct Adam8Args {
  Seg8 seg[kMaxLayersPerLaunch];
  int n_seg;
  uint32_t k0, k1, step;     // noise
  uint32_t r0, r1, t;        // rounding
  float sigmaC, scale;
  float beta1, beta2, one_m_beta1, one_m_beta2;
  float step_size, inv_sqrt_bc2, eps, decay;
};

template <class Args>
__device__ __forceinline__ const auto& seg_of(const Args& a, uint32_t wg) {
  int lo = 0, hi = a.n_seg - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seg[mid].wg_begin <= wg) lo = mid; else hi = mid - 1;
  }
  return a.seg[lo];
}

// Four entries from e on, 0 past the end (n entries).
__device__ __forceinline__ void load4(const float* p, int64_t e, int64_t n, float (&x)[4]) {
  if (e + 4 <= n) {
    const f32x4_t q = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p + e));
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = q[c];
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = e + c < n ? p[e + c] : 0.0f;
  }
}

__device__ __forceinline__ void store4(float* p, int64_t e, int64_t n, const float (&x)[4]) {
  if (e + 4 <= n) {
    __builtin_nontemporal_store(f32x4_t{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4_t*>(p + e));
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (e + c < n) p[e + c] = x[c];
  }
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t e, int64_t n) {
  if (e + 4 <= n) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p + e));
  uint32_t w = 0;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (e + c < n) w |= (uint32_t)p[e + c] << (8 * c);
  return w;
}

__device__ __forceinline__ void store_codes(uint8_t* p, int64_t e, int64_t n, uint32_t w) {
  if (e + 4 <= n) {
    __builtin_nontemporal_store(w, reinterpret_cast<uint32_t*>(p + e));
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (e + c < n) p[e + c] = (uint8_t)(w >> (8 * c));
  }
}

__device__ __forceinline__ uint32_t largest_bits(const float (&x)[4]) {
  uint32_t b = 0;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t u = __float_as_uint(x[c]) & 0x7FFFFFFFu;
    b = u > b ? u : b;
  }
  return b;
}

template <bool STOCHASTIC, int kBlocksPerWave>
__global__ __launch_bounds__(kThreads) void noise_adamw8_kernel(Adam8Args a) {
  const Seg8& s = seg_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63;
  const int64_t first = ((int64_t)(blockIdx.x - s.wg_begin) * (kThreads / 64) + (threadIdx.x >> 6)) *
                        kBlocksPerWave;
  const int64_t n = s.numel;
  const bool with_noise = a.sigmaC != 0.0f;

  float S[kBlocksPerWave][4], p[kBlocksPerWave][4];
  uint32_t qm[kBlocksPerWave], qv[kBlocksPerWave], k[kBlocksPerWave];
#pragma unroll
  for (int u = 0; u < kBlocksPerWave; ++u) {
    const int64_t e = (first + u) * kStateBlock + lane * 4;
    load4(s.grad, e, n, S[u]);
    load4(s.param, e, n, p[u]);
    qm[u] = load_codes(s.m, e, n);
    qv[u] = load_codes(s.v, e, n);
    k[u] = (first + u) * kStateBlock < n
               ? *reinterpret_cast<const uint16_t*>(s.exps + (first + u) * 2) : 0u;
  }
#pragma unroll
  for (int u = 0; u < kBlocksPerWave; ++u) {
    if ((first + u) * kStateBlock >= n) break;   // the whole wave
    const int64_t e = (first + u) * kStateBlock + lane * 4;
    const uint64_t j = (uint64_t)(e >> 2);
    float z[4] = {};
    if (with_noise) {
      const float4 q = normals_of_block(j, s.tensor_id, a.step, a.k0, a.k1);
      z[0] = q.x;
      z[1] = q.y;
      z[2] = q.z;
      z[3] = q.w;
    }
    float m[4], v[4], g[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool in = e + c < n;
      const float m0 = value_m((qm[u] >> (8 * c)) & 255u, k[u] & 255u);
      const float v0 = value_v((qv[u] >> (8 * c)) & 255u, k[u] >> 8);
      g[c] = a.scale * (with_noise ? fmaf(a.sigmaC, z[c], S[u][c]) : S[u][c]);
      m[c] = a.beta1 * m0 + a.one_m_beta1 * g[c];
      v[c] = a.beta2 * v0 + a.one_m_beta2 * (g[c] * g[c]);
      const float denom = sqrtf(v[c]) * a.inv_sqrt_bc2 + a.eps;
      p[u][c] = p[u][c] * a.decay - (m[c] / denom) * a.step_size;
      if (!in) m[c] = v[c] = 0.0f;
    }
    const uint32_t km = block_exponent(wave_max_u32(largest_bits(m)), kLowM);
    const uint32_t kv = block_exponent(wave_max_u32(largest_bits(v)), kLowV);
    uint32_t r[4] = {};
    if constexpr (STOCHASTIC) {
      const uint4 w = philox4x32_10((uint32_t)j, (uint32_t)(j >> 32), s.tensor_id, a.t, a.r0, a.r1);
      r[0] = w.x;
      r[1] = w.y;
      r[2] = w.z;
      r[3] = w.w;
    }
    store4(s.param, e, n, p[u]);
    if (s.noisy) store4(s.noisy, e, n, g);
    store_codes(s.m, e, n, codes_m<STOCHASTIC>(m, km, r));
    store_codes(s.v, e, n, codes_v<STOCHASTIC>(v, kv, r));
    if (lane == 0) *reinterpret_cast<uint16_t*>(s.exps + (first + u) * 2) = (uint16_t)(km | kv << 8);
  }
}

__global__ __launch_bounds__(kThreads) void adamw8_pack_kernel(Adam8Args a) {
  constexpr int kBlocksPerWave = kManyBlocks;
  const Seg8& s = seg_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63;
  const int64_t first = ((int64_t)(blockIdx.x - s.wg_begin) * (kThreads / 64) + (threadIdx.x >> 6)) *
                        kBlocksPerWave;
  const int64_t n = s.numel;
  const uint32_t none[4] = {};
  for (int u = 0; u < kBlocksPerWave; ++u) {
    if ((first + u) * kStateBlock >= n) break;
    const int64_t e = (first + u) * kStateBlock + lane * 4;
    float m[4], v[4];
    load4(s.grad, e, n, m);
    load4(s.param, e, n, v);
    bool negative = false;
#pragma unroll
    for (int c = 0; c < 4; ++c) negative = negative || v[c] < 0.0f;
    const uint32_t km = block_exponent(wave_max_u32(largest_bits(m)), kLowM);
    uint32_t kv = block_exponent(wave_max_u32(largest_bits(v)), kLowV);
    if (__any(negative)) kv = kNotFinite;
    store_codes(s.m, e, n, codes_m<false>(m, km, none));
    store_codes(s.v, e, n, codes_v<false>(v, kv, none));
    if (lane == 0) *reinterpret_cast<uint16_t*>(s.exps + (first + u) * 2) = (uint16_t)(km | kv << 8);
  }
}

struct UnpackSeg {
  const uint8_t* m;
  const uint8_t* v;
  const uint8_t* exps;
  void* m_out;
  void* v_out;
  int64_t numel;
  uint32_t wg_begin;
};

struct UnpackArgs {
  UnpackSeg seg[kMaxLayersPerLaunch];
  int n_seg;
};

template <class T>
__device__ __forceinline__ void store_values(T* p, int64_t e, int64_t n, const float (&x)[4]) {
  if (e + 4 <= n) {
    store_vec<4>(p + e, x);
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float one[1] = {x[c]};
      if (e + c < n) store_vec<1>(p + e + c, one);
    }
  }
}

template <class T, int kBlocksPerWave>
__global__ __launch_bounds__(kThreads) void adamw8_unpack_kernel(UnpackArgs a) {
  const UnpackSeg& s = seg_of(a, blockIdx.x);
  const int lane = threadIdx.x & 63;
  const int64_t first = ((int64_t)(blockIdx.x - s.wg_begin) * (kThreads / 64) + (threadIdx.x >> 6)) *
                        kBlocksPerWave;
  const int64_t n = s.numel;
  uint32_t qm[kBlocksPerWave], qv[kBlocksPerWave], k[kBlocksPerWave];
#pragma unroll
  for (int u = 0; u < kBlocksPerWave; ++u) {
    const int64_t e = (first + u) * kStateBlock + lane * 4;
    qm[u] = load_codes(s.m, e, n);
    qv[u] = load_codes(s.v, e, n);
    k[u] = (first + u) * kStateBlock < n
               ? *reinterpret_cast<const uint16_t*>(s.exps + (first + u) * 2) : 0u;
  }
#pragma unroll
  for (int u = 0; u < kBlocksPerWave; ++u) {
    const int64_t e = (first + u) * kStateBlock + lane * 4;
    float m[4], v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      m[c] = value_m((qm[u] >> (8 * c)) & 255u, k[u] & 255u);
      v[c] = value_v((qv[u] >> (8 * c)) & 255u, k[u] >> 8);
    }
    store_values(static_cast<T*>(s.m_out), e, n, m);
    store_values(static_cast<T*>(s.v_out), e, n, v);
  }
}

int64_t wgs_of(int64_t numel, int per_wave) {
  return ceil_div(ceil_div(numel, kStateBlock), blocks_per_wg(per_wave));
}

// Blocks of a wave for a launch over n tensors.
int blocks_per_wave(const dpsgd_layer* layers, int n) {
  int64_t blocks = 0;
  for (int l = 0; l < n; ++l) blocks += ceil_div(layers[l].d_out * layers[l].d_in, kStateBlock);
  return blocks <= kFewBlocks ? 1 : kManyBlocks;
}

// Whether each of a call's launches can be: asked before the first, so that a call that is
// refused has changed nothing. (Launches of few blocks a wave are small.)
bool all_launchable(const dpsgd_layer* layers, int n_layers) {
  for (int base = 0; base < n_layers; base += kMaxLayersPerLaunch) {
    int64_t wgs = 0;
    for (int l = base; l < n_layers && l < base + kMaxLayersPerLaunch; ++l)
      wgs += wgs_of(layers[l].d_out * layers[l].d_in, kManyBlocks);
    if (!launchable(wgs, kThreads)) return false;
  }
  return true;
}

}  // namespace

int launch_noise_adamw8(const dpsgd_layer* layers, int n_layers, const float* const* grads,
                        float* const* params, uint8_t* const* ms, uint8_t* const* vs,
                        uint8_t* const* exps, float* const* noisy, float sigma, float C,
                        uint64_t seed, uint32_t step, float scale, const dpsgd_adamw& opt,
                        int32_t rounding, uint64_t round_seed, hipStream_t stream) {
  if (!all_launchable(layers, n_layers)) return DPSGD_ERR_INVALID_ARG;
  const double bc1 = 1.0 - pow((double)opt.beta1, (double)opt.t);
  const double bc2 = 1.0 - pow((double)opt.beta2, (double)opt.t);
  for (int base = 0; base < n_layers; base += kMaxLayersPerLaunch) {
    const int n = n_layers - base < kMaxLayersPerLaunch ? n_layers - base : kMaxLayersPerLaunch;
    Adam8Args args{};
    args.n_seg = n;
    args.k0 = (uint32_t)seed;
    args.k1 = (uint32_t)(seed >> 32);
    args.step = step;
    args.r0 = (uint32_t)~round_seed;
    args.r1 = (uint32_t)(~round_seed >> 32);
    args.t = opt.t;
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
    const int per_wave = blocks_per_wave(layers + base, n);
    int64_t wgs = 0;
    for (int l = 0; l < n; ++l) {
      const dpsgd_layer& L = layers[base + l];
      args.seg[l] = Seg8{grads[base + l], params[base + l], ms[base + l], vs[base + l],
                         exps[base + l], noisy ? noisy[base + l] : nullptr, L.d_out * L.d_in,
                         L.tensor_id, (uint32_t)wgs};
      wgs += wgs_of(L.d_out * L.d_in, per_wave);
    }
    const dim3 grid((uint32_t)wgs), block(kThreads);
    if (rounding == DPSGD_ROUND_STOCHASTIC && per_wave == 1)
      hipLaunchKernelGGL((noise_adamw8_kernel<true, 1>), grid, block, 0, stream, args);
    else if (rounding == DPSGD_ROUND_STOCHASTIC)
      hipLaunchKernelGGL((noise_adamw8_kernel<true, kManyBlocks>), grid, block, 0, stream, args);
    else if (per_wave == 1)
      hipLaunchKernelGGL((noise_adamw8_kernel<false, 1>), grid, block, 0, stream, args);
    else
      hipLaunchKernelGGL((noise_adamw8_kernel<false, kManyBlocks>), grid, block, 0, stream, args);
    if (check_launch() != DPSGD_OK) return DPSGD_ERR_HIP;
  }
  return DPSGD_OK;
}

int launch_adamw8_pack(const dpsgd_layer* layers, int n_layers, const float* const* ms_in,
                       const float* const* vs_in, uint8_t* const* ms, uint8_t* const* vs,
                       uint8_t* const* exps, hipStream_t stream) {
  if (!all_launchable(layers, n_layers)) return DPSGD_ERR_INVALID_ARG;
  for (int base = 0; base < n_layers; base += kMaxLayersPerLaunch) {
    const int n = n_layers - base < kMaxLayersPerLaunch ? n_layers - base : kMaxLayersPerLaunch;
    Adam8Args args{};
    args.n_seg = n;
    int64_t wgs = 0;
    for (int l = 0; l < n; ++l) {
      const dpsgd_layer& L = layers[base + l];
      args.seg[l] = Seg8{ms_in[base + l], const_cast<float*>(vs_in[base + l]), ms[base + l],
                         vs[base + l], exps[base + l], nullptr, L.d_out * L.d_in, 0, (uint32_t)wgs};
      wgs += wgs_of(L.d_out * L.d_in, kManyBlocks);
    }
    hipLaunchKernelGGL(adamw8_pack_kernel, dim3((uint32_t)wgs), dim3(kThreads), 0, stream, args);
    if (check_launch() != DPSGD_OK) return DPSGD_ERR_HIP;
  }
  return DPSGD_OK;
}

int launch_adamw8_unpack(const dpsgd_layer* layers, int n_layers, const uint8_t* const* ms,
                         const uint8_t* const* vs, const uint8_t* const* exps, void* const* ms_out,
                         void* const* vs_out, int32_t out_dtype, hipStream_t stream) {
  if (!all_launchable(layers, n_layers)) return DPSGD_ERR_INVALID_ARG;
  for (int base = 0; base < n_layers; base += kMaxLayersPerLaunch) {
    const int n = n_layers - base < kMaxLayersPerLaunch ? n_layers - base : kMaxLayersPerLaunch;
    UnpackArgs args{};
    args.n_seg = n;
    const int per_wave = blocks_per_wave(layers + base, n);
    int64_t wgs = 0;
    for (int l = 0; l < n; ++l) {
      const dpsgd_layer& L = layers[base + l];
      args.seg[l] = UnpackSeg{ms[base + l], vs[base + l], exps[base + l], ms_out[base + l],
                              vs_out[base + l], L.d_out * L.d_in, (uint32_t)wgs};
      wgs += wgs_of(L.d_out * L.d_in, per_wave);
    }
    const dim3 grid((uint32_t)wgs), block(kThreads);
    if (out_dtype == DPSGD_BF16 && per_wave == 1)
      hipLaunchKernelGGL((adamw8_unpack_kernel<uint16_t, 1>), grid, block, 0, stream, args);
    else if (out_dtype == DPSGD_BF16)
      hipLaunchKernelGGL((adamw8_unpack_kernel<uint16_t, kManyBlocks>), grid, block, 0, stream, args);
    else if (per_wave == 1)
      hipLaunchKernelGGL((adamw8_unpack_kernel<float, 1>), grid, block, 0, stream, args);
    else
      hipLaunchKernelGGL((adamw8_unpack_kernel<float, kManyBlocks>), grid, block, 0, stream, args);
    if (check_launch() != DPSGD_OK) return DPSGD_ERR_HIP;
  }
  return DPSGD_OK;
}

}  // namespace dpsgd
