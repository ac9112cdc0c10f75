// Activations of the layer operators and their derivatives, in fp32, and
// bf16 packing.
//
// gelu uses the error function through the rational form 7.1.26 of
// Abramowitz and Stegun, Handbook of Mathematical Functions: erfc(x) =
// (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x), x >= 0, absolute error
// below 1.5e-7 — at the level of fp32 rounding of the result — with one
// exponential that the derivative's density term shares.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

#include "../../include/goldy.h"

namespace goldy {

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return uint32_t(__bfloat16_as_ushort(h.x)) | (uint32_t(__bfloat16_as_ushort(h.y)) << 16);
}
__device__ __forceinline__ float load_bf16(const void* p, int64_t i) {
  return __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[i]) << 16);
}
__device__ __forceinline__ void store_bf16(void* p, int64_t i, float v) {
  static_cast<uint16_t*>(p)[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  f[0] = bf16_lo(v.x), f[1] = bf16_hi(v.x), f[2] = bf16_lo(v.y), f[3] = bf16_hi(v.y);
  f[4] = bf16_lo(v.z), f[5] = bf16_hi(v.z), f[6] = bf16_lo(v.w), f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

// Standard normal upper tail q(|z|) = erfc(|z| / sqrt 2) / 2 and density
// factor g = exp(-z^2 / 2).
__device__ __forceinline__ float normal_tail(float z, float& g) {
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = __fdividef(1.0f, fmaf(0.3275911f, x, 1.0f));
  g = __expf(-x * x);
  float s = fmaf(1.061405429f, t, -1.453152027f);
  s = fmaf(s, t, 1.421413741f);
  s = fmaf(s, t, -0.284496736f);
  s = fmaf(s, t, 0.254829592f);
  return 0.5f * s * t * g;
}

__device__ __forceinline__ float act_value(float z, int act) {
  switch (act) {
    case GOLDY_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case GOLDY_ACT_GELU: {
      float g;
      const float q = normal_tail(z, g);
      return z * (z < 0.0f ? q : 1.0f - q);
    }
    case GOLDY_ACT_GELU_TANH: {
      // (1 + tanh u) / 2 = 1 / (1 + exp(-2u)), u = sqrt(2/pi) (z + 0.044715 z^3)
      const float u2 = 1.5957691216057308f * fmaf(0.044715f * z * z, z, z);
      return __fdividef(z, 1.0f + __expf(-u2));
    }
    case GOLDY_ACT_SILU: return __fdividef(z, 1.0f + __expf(-z));
    default: return z;
  }
}

__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case GOLDY_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case GOLDY_ACT_GELU: {
      float g;
      const float q = normal_tail(z, g);
      return fmaf(z * 0.39894228040143268f, g, z < 0.0f ? q : 1.0f - q);
    }
    case GOLDY_ACT_GELU_TANH: {
      const float zz = fminf(z * z, 1e30f);      // finite, so that a saturated slope stays 0 or 1
      const float u2 = 1.5957691216057308f * fmaf(0.044715f * zz, z, z);
      const float s = __fdividef(1.0f, 1.0f + __expf(-u2));
      return fmaf(z * s * (1.0f - s), 1.5957691216057308f * fmaf(3.0f * 0.044715f, zz, 1.0f), s);
    }
    case GOLDY_ACT_SILU: {
      const float s = __fdividef(1.0f, 1.0f + __expf(-z));
      return s * fmaf(z, 1.0f - s, 1.0f);
    }
    default: return 1.0f;
  }
}

}  // namespace goldy
