// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC'11) and the Box-Muller (1958)
// normals that are formed from its blocks.
#pragma once

#include "common.h"

namespace dpsgd {

constexpr uint32_t kPhiloxM0 = 0xD2511F53u;
constexpr uint32_t kPhiloxM1 = 0xCD9E8D57u;
constexpr uint32_t kWeyl0 = 0x9E3779B9u;
constexpr uint32_t kWeyl1 = 0xBB67AE85u;

__device__ __forceinline__ uint4 philox4x32_10(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3,
                                               uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)x0 * kPhiloxM0;
    const uint64_t p1 = (uint64_t)x2 * kPhiloxM1;
    const uint32_t n0 = (uint32_t)(p1 >> 32) ^ x1 ^ k0;
    const uint32_t n2 = (uint32_t)(p0 >> 32) ^ x3 ^ k1;
    x1 = (uint32_t)p1;
    x3 = (uint32_t)p0;
    x0 = n0;
    x2 = n2;
    k0 += kWeyl0;
    k1 += kWeyl1;
  }
  return make_uint4(x0, x1, x2, x3);
}

// Four standard normals from one block: lanes (0,1) from (r0,r1), (2,3) from (r2,r3).
// u in (0,1] and v in [0,1) are exact; sin/cos take their argument in turns.
__device__ __forceinline__ float4 box_muller4(uint4 r) {
  const float ua = (float)((r.x >> 8) + 1u) * 0x1p-24f;
  const float va = (float)(r.y >> 8) * 0x1p-24f;
  const float ub = (float)((r.z >> 8) + 1u) * 0x1p-24f;
  const float vb = (float)(r.w >> 8) * 0x1p-24f;
  const float ra = sqrtf(-2.0f * logf(ua));
  const float rb = sqrtf(-2.0f * logf(ub));
  return make_float4(ra * __builtin_amdgcn_cosf(va), ra * __builtin_amdgcn_sinf(va),
                     rb * __builtin_amdgcn_cosf(vb), rb * __builtin_amdgcn_sinf(vb));
}

__device__ __forceinline__ float4 normals_of_block(uint64_t j, uint32_t tensor_id, uint32_t step,
                                                    uint32_t k0, uint32_t k1) {
  return box_muller4(philox4x32_10((uint32_t)j, (uint32_t)(j >> 32), tensor_id, step, k0, k1));
}

}  // namespace dpsgd
