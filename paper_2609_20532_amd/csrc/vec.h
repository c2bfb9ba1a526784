// Loads and stores of a few consecutive elements as float32: float or bf16
// (uint16_t bits, rounded to nearest-even on the way out).
#pragma once

#include "common.h"

namespace dpsgd {

// Elements p[0..V) widened to float32. p is aligned to min(16, V sizeof(T)) bytes.
template <int V>
__device__ __forceinline__ void load_vec(const float* p, float (&x)[V]) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int k = 0; k < V; k += 4) {
      const f32x4_t q = *reinterpret_cast<const f32x4_t*>(p + k);
#pragma unroll
      for (int c = 0; c < 4; ++c) x[k + c] = q[c];
    }
  } else if constexpr (V == 2) {
    const float2 q = *reinterpret_cast<const float2*>(p);
    x[0] = q.x;
    x[1] = q.y;
  } else {
    x[0] = *p;
  }
}

template <int V>
__device__ __forceinline__ void load_vec(const uint16_t* p, float (&x)[V]) {
  if constexpr (V == 8) {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      x[2 * c] = bf16_lo(w[c]);
      x[2 * c + 1] = bf16_hi(w[c]);
    }
  } else if constexpr (V == 4) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    x[0] = bf16_lo(q.x);
    x[1] = bf16_hi(q.x);
    x[2] = bf16_lo(q.y);
    x[3] = bf16_hi(q.y);
  } else if constexpr (V == 2) {
    const uint32_t q = *reinterpret_cast<const uint32_t*>(p);
    x[0] = bf16_lo(q);
    x[1] = bf16_hi(q);
  } else {
    x[0] = bf16_to_f32(*p);
  }
}

template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&x)[V]) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int k = 0; k < V; k += 4)
      *reinterpret_cast<f32x4_t*>(p + k) = f32x4_t{x[k], x[k + 1], x[k + 2], x[k + 3]};
  } else if constexpr (V == 2) {
    *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
  } else {
    *p = x[0];
  }
}

template <int V>
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&x)[V]) {
  if constexpr (V == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                              pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  } else if constexpr (V == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  } else if constexpr (V == 2) {
    *reinterpret_cast<uint32_t*>(p) = pack_bf16x2(x[0], x[1]);
  } else {
    *p = (uint16_t)pack_bf16x2(x[0], 0.0f);
  }
}

// The same elements as they lie in memory, in registers: for loads that stay in
// flight while others are issued.
template <class T, int V>
struct Raw {
  static constexpr int kBytes = V * (int)sizeof(T);
  uint32_t w[kBytes >= 4 ? kBytes / 4 : 1];

  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int k = 0; k < kBytes / 16; ++k) {
        const uint4 q = reinterpret_cast<const uint4*>(p)[k];
        w[4 * k] = q.x;
        w[4 * k + 1] = q.y;
        w[4 * k + 2] = q.z;
        w[4 * k + 3] = q.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      w[0] = q.x;
      w[1] = q.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& x : w) x = 0;
  }

  // Keeps the compiler from holding on to what was formed from these elements
  // before: later uses form it again, and only the elements stay in registers.
  __device__ __forceinline__ void keep_raw() {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (uint32_t& x : w) asm volatile("" : "+v"(x));
    }
  }

  __device__ __forceinline__ void widen(float (&x)[V]) const {
#pragma unroll
    for (int c = 0; c < V; ++c) {
      if constexpr (sizeof(T) == 4)
        x[c] = __uint_as_float(w[c]);
      else
        x[c] = c & 1 ? bf16_hi(w[c / 2]) : bf16_lo(w[c / 2]);
    }
  }
};

// Largest of 8, 4, 2, 1 (at most `most`) that divides n.
inline int vec_width(int64_t n, int most) {
  for (int v = most; v > 1; v >>= 1)
    if (n % v == 0) return v;
  return 1;
}

// Sum over the lanes of a wave in every lane, in a fixed order: shifts within rows
// of 16 lanes, then the rows' last lanes to the rows after them (no LDS).
__device__ __forceinline__ float wave_total(float v) {
#define DPSGD_DPP(ctrl, rows) \
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
  DPSGD_DPP(0x111, 0xf);   // row_shr 1, 2, 4, 8
  DPSGD_DPP(0x112, 0xf);
  DPSGD_DPP(0x114, 0xf);
  DPSGD_DPP(0x118, 0xf);
  DPSGD_DPP(0x142, 0xa);   // row_bcast 15, 31
  DPSGD_DPP(0x143, 0xc);
#undef DPSGD_DPP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// n / d for n < 2^31, by the magic and shift of divide_magic.
__device__ __forceinline__ uint32_t magic_divide(uint32_t n, uint32_t magic, int32_t shift) {
  return shift < 0 ? n : __umulhi(n, magic) >> shift;
}

}  // namespace dpsgd
