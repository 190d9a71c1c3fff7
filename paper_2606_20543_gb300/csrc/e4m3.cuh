// e4m3.cuh — e4m3 (4 exponent bits, 3 mantissa bits, largest value 448) as the cache and the
// quantised products hold it, and what both read and write.
#pragma once

#include <cuda_fp8.h>

#include "kernels.cuh"

namespace ssd {

constexpr float kTop8 = 448.f;       // largest e4m3 value
constexpr float kLeast = 0x1p-100f;  // least magnitude a block is scaled by

__device__ __forceinline__ void unpack8(const uint4& w, float* x) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                    pack_bf16x2(x[6], x[7]));
}
// Two float32 to e4m3, to nearest even; +-448 beyond, NaN for NaN.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 to_e4m3x8(const float* x, float f) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = to_e4m3x2(x[2 * i] * f, x[2 * i + 1] * f);
  return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}
__device__ __forceinline__ float2 from_e4m3x2(uint16_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(w));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

}  // namespace ssd
