// Numbers -> codes of the 8-bit paged cache: a block's scale, rounding to it, and rounding again when it grows.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "paged.cuh"

namespace skv {

template <int FMT>
__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
  if (amax_bits == 0) return 0.f;
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
    return fmaxf(__fdiv_rn(__uint_as_float(amax_bits), 127.f), 1.17549435e-38f);
  } else {
    // amax = 1.m 2^(e-127): least k with 1.m 2^(e-127) <= 1.75 2^(8+k)
    const int e = (int)(amax_bits >> 23);
    const int k = max(e - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), -126);
    return __uint_as_float((uint32_t)(k + 127) << 23);
  }
}

// inv: 1 / s (exact for E4M3)
__device__ __forceinline__ int round_int8(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), half = 0.5f * s;
  const float up = r > 0.f ? 1.f : -1.f;
  const bool odd = ((int)q & 1) != 0;
  if (fabsf(r) > half || (fabsf(r) == half && odd)) q += up;
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}

// low bytes of eight words
__device__ __forceinline__ uint2 low_bytes(const uint32_t (&t)[8]) {
  return make_uint2(__byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410));
}

// worst: the largest |x - code * s| so far (int8)
template <int FMT>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float s, float inv, float& worst) {
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float sum = fmaf(x[i], inv, 12582912.f);
      t[i] = __float_as_uint(sum);
      worst = fmaxf(worst, fabsf(fmaf(12582912.f - sum, s, x[i])));
    }
    return low_bytes(t);
  } else {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i] * inv, x[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      w[i >> 1] |= two << (16 * (i & 1));
    }
    return make_uint2(w[0], w[1]);
  }
}
__device__ __forceinline__ uint2 encode8_exactly(const float (&x)[8], float s, float inv) {
  uint32_t t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = (uint32_t)round_int8(x[i], s, inv);
  return low_bytes(t);
}

// codes at scale `was` -> codes at the larger scale `s`
template <int FMT>
__device__ __forceinline__ uint2 recode8(uint2 c, float was, float s) {
  const uint32_t in[2] = {c.x, c.y};
  uint32_t w[2] = {0u, 0u};
  if constexpr (FMT == SPINDLEKV_PAGED_INT8) {
    // code * was has up to 31 bits: in double, where the product is exact and the quotient's rounding cannot reach a tie
    // that the exact quotient does not have
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int v = (int)(int8_t)(in[i >> 2] >> (8 * (i & 3)));
      const int q = (int)rint((double)v * (double)was / (double)s);
      w[i >> 2] |= (uint32_t)(q & 0xFF) << (8 * (i & 3));
    }
  } else {
    const float f = __fdiv_rn(was, s);   // a power of two; what falls below the smallest fp32 number falls below E4M3's too
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(in[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
      const float2 v = __half22float2(__half2(h));
      const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(v.x * f, v.y * f), __NV_SATFINITE, __NV_E4M3);
      w[i >> 1] |= two << (16 * (i & 1));
    }
  }
  return make_uint2(w[0], w[1]);
}

}  // namespace skv
