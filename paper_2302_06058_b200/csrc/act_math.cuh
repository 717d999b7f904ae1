// Arithmetic shared by the linear-layer kernels: the activations and their derivatives, and the 8-bit activation
// checkpoint (32 consecutive channels of a token = one block of signed bytes q and one scale byte s, values
// q 2^(s - 127)).  Everything is evaluated in fp32.
#pragma once
#include "common.cuh"
#include <cuda_bf16.h>

namespace bimask {
namespace act {

// 2^x and 1/x by the special-function unit (about 2 and 1 ulp): errors of 1e-7 relative, far below the rounding to
// bf16 and within what fp32 column sums of the results need.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// larger / smaller of two numbers, NaN if either is one
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

constexpr float LOG2E = 1.4426950408889634f;
constexpr float GELU_C = 0.7978845608028654f;            // sqrt(2 / pi)
constexpr float GELU_A = 0.044715f;
constexpr float INV_SQRT_2PI = 0.3989422804014327f;

// sigma(x) = 1 / (1 + e^-x); e^-x = inf for very negative x gives 0
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.0f + ex2(-LOG2E * x)); }

// Phi(z) = erfc(-z / sqrt 2) / 2 by formula 7.1.26 of Abramowitz and Stegun: with x = |z| / sqrt 2 and
// t = 1 / (1 + 0.3275911 x), erfc(x) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) e^(-x^2) to 1.5e-7.  The factor
// e^(-z^2 / 2) is handed back too: it is the density's.
__device__ __forceinline__ float normal_cdf(float z, float& gauss) {
  const float a = fabsf(z);
  const float t = rcp(fmaf(0.3275911f * 0.7071067811865476f, a, 1.0f));
  gauss = ex2(-0.5f * LOG2E * z * z);
  float p = fmaf(1.061405429f * 0.5f, t, -1.453152027f * 0.5f);
  p = fmaf(p, t, 1.421413741f * 0.5f);
  p = fmaf(p, t, -0.284496736f * 0.5f);
  p = fmaf(p, t, 0.254829592f * 0.5f);
  const float tail = p * t * gauss;                       // Phi(-|z|)
  return z < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float relu(float z) { return z > 0.0f ? z : (z != z ? z : 0.0f); }
__device__ __forceinline__ float gelu(float z) { float g; return z * normal_cdf(z, g); }
__device__ __forceinline__ float gelu_tanh(float z) {     // z (1 + tanh u) / 2 = z sigma(2 u), u = c (z + a z^3)
  return z * sigmoid(2.0f * GELU_C * z * fmaf(GELU_A * z, z, 1.0f));
}
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }

__device__ __forceinline__ float relu_slope(float z) { return z > 0.0f ? 1.0f : (z != z ? z : 0.0f); }
__device__ __forceinline__ float gelu_slope(float z) {
  float g;
  const float c = normal_cdf(z, g);
  return fmaf(INV_SQRT_2PI * g, z, c);
}
__device__ __forceinline__ float gelu_tanh_slope(float z) {
  z = min_nan(max_nan(z, -16.0f), 16.0f);                 // 0 and 1 to fp32 beyond: keeps z^2 times 0 finite
  const float s = sigmoid(2.0f * GELU_C * z * fmaf(GELU_A * z, z, 1.0f));
  return fmaf(z * s * (1.0f - s), 2.0f * GELU_C * fmaf(3.0f * GELU_A * z, z, 1.0f), s);
}
__device__ __forceinline__ float silu_slope(float z) {
  z = min_nan(max_nan(z, -128.0f), 128.0f);
  const float s = sigmoid(z);
  return s * fmaf(z, 1.0f - s, 1.0f);
}

// f over an array, the activation chosen once for all of it
template <int N>
__device__ __forceinline__ void apply(int kind, float (&z)[N]) {
  switch (kind) {
    case BIMASK_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = relu(z[i]);
      break;
    case BIMASK_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = gelu(z[i]);
      break;
    case BIMASK_ACT_GELU_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = gelu_tanh(z[i]);
      break;
    case BIMASK_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = silu(z[i]);
      break;
    default: break;
  }
}

template <int KIND>
__device__ __forceinline__ float value(float z) {
  return KIND == BIMASK_ACT_RELU ? relu(z) : KIND == BIMASK_ACT_GELU ? gelu(z) : KIND == BIMASK_ACT_GELU_TANH ? gelu_tanh(z)
         : KIND == BIMASK_ACT_SILU ? silu(z) : z;
}
template <int KIND>
__device__ __forceinline__ float slope(float z) {
  return KIND == BIMASK_ACT_RELU ? relu_slope(z) : KIND == BIMASK_ACT_GELU ? gelu_slope(z)
         : KIND == BIMASK_ACT_GELU_TANH ? gelu_tanh_slope(z) : KIND == BIMASK_ACT_SILU ? silu_slope(z) : 1.0f;
}

}  // namespace act

// ---- 8-bit checkpoint ---------------------------------------------------------------------------
namespace ckpt {

// The scale depends on max |x| only through the comparison with 127 * 2^e, whose mantissa ends within the seven bits of
// a bf16: so the maximum may be taken on |x| rounded UP to bf16, 16 bits that compare as integers (NaN above infinity
// above every finite value).
__device__ __forceinline__ uint32_t up16(float abs_x) { return (__float_as_uint(abs_x) + 0xFFFFu) >> 16; }

// Scale byte of a block from that maximum h: 2^(s-127) is the smallest power of two, not below 2^-126, with
// max |x| <= 127 * 2^(s-127); 255: the block holds a value that is not finite in bf16.
__device__ __forceinline__ uint32_t scale_of(uint32_t h) {
  const int s = (int)((h + 1u) >> 7) - 6;                 // exponent of h, one more when its mantissa is above 1.984375 = 127 / 64
  return h >= 0x7F80u ? 255u : (uint32_t)(s < 1 ? 1 : s);
}
// 2^(127 - s): x times it is exact, and rounds to the byte
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127); NaN for 255
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s == 255u ? 0x7FC00000u : s << 23); }

// Round x / 2^(s-127) to the nearest integer (ties to even): it is the low byte of the result's bits.
__device__ __forceinline__ uint32_t round_bits(float x, float inv) { return __float_as_uint(fmaf(x, inv, 12582912.0f)); }

// bytes 0..3 of w as fp32 integers times the scale.  The byte plus 128 goes into the low bits of 2^23: exact.
__device__ __forceinline__ void decode4(uint32_t w, float scale, float* out) {
  const uint32_t u = w ^ 0x80808080u;
  const float bias = -8388736.0f;                         // -(2^23 + 128)
  out[0] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540)) + bias) * scale;
  out[1] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7541)) + bias) * scale;
  out[2] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7542)) + bias) * scale;
  out[3] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7543)) + bias) * scale;
}

}  // namespace ckpt

__device__ __forceinline__ uint32_t pack_bf16_f(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

}  // namespace bimask
