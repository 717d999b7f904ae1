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

// The largest of three magnitudes, NaN if any is one.
__device__ __forceinline__ float max_abs3(float a, float b, float c) {
  float y;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// Two fp32 numbers in one register pair: one instruction for both, each rounded as by the scalar one.
struct Pair { unsigned long long v; };
__device__ __forceinline__ Pair pair(float lo, float hi) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ Pair both(float x) { return pair(x, x); }
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p.v)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
template <typename F>
__device__ __forceinline__ Pair map2(Pair a, F f) {
  float x, y;
  split(a, x, y);
  return pair(f(x), f(y));
}

constexpr float LOG2E = 1.4426950408889634f;
constexpr float GELU_C = 0.7978845608028654f;            // sqrt(2 / pi)
constexpr float GELU_A = 0.044715f;
constexpr float INV_SQRT_2PI = 0.3989422804014327f;

// Both GELUs are z times a distribution function F with F(-a) = 1 - F(a), so
//   z F(z) = max(z, 0) - a t(a),   a = |z|,  t(a) = F(-a),
// and log2 t is smooth: t = 2^P(a) with a polynomial P, one special-function operation where e^x and a reciprocal (or
// an error function) would take two and more.  P is the minimax fit of a t(a) (of 0.3 t(a) below a = 0.3, which keeps
// small results exact in their leading digits), by linear programming on a dense grid, held near log2 t further out and
// below -127 at CUT, where a is cut off: there 2^P is flushed to 0, and infinity times 0 cannot arise.  The error of
// a t(a) in fp32 is 1.5e-7 (normal, degree 6) and 2.5e-7 (tanh form, degree 8).
struct NormalTail {                                       // t(a) = erfc(a / sqrt 2) / 2
  static constexpr float CUT = 13.5f;
  static constexpr int N = 7;
  static __device__ __forceinline__ constexpr float c(int i) {
    constexpr float k[N] = {-1.00000101f, -1.15111779f, -0.459027313f, -0.0530767738f, 0.00787010158f, -0.00070691381f, 2.61608362e-05f};
    return k[i];
  }
};
struct TanhTail {                                         // t(a) = (1 - tanh(c (a + 0.044715 a^3))) / 2
  static constexpr float CUT = 9.4f;
  static constexpr int N = 9;
  static __device__ __forceinline__ constexpr float c(int i) {
    constexpr float k[N] = {-0.999997816f, -1.15116158f, -0.459060495f, -0.0511946513f, 0.00609492494f, 0.00223345144f,
                            -0.00187715303f, 0.000335500797f, -1.86449501e-05f};
    return k[i];
  }
};
template <typename T>
__device__ __forceinline__ float tail(float a) {          // a in [0, CUT]
  float p = T::c(T::N - 1);
#pragma unroll
  for (int i = T::N - 2; i >= 0; --i) p = fmaf(p, a, T::c(i));
  return ex2(p);
}
template <typename T>
__device__ __forceinline__ float cut(float z) { return min_nan(fabsf(z), T::CUT); }

// sigma(x) = 1 / (1 + e^-x); e^-x = inf for very negative x gives 0
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.0f + ex2(-LOG2E * x)); }

__device__ __forceinline__ float relu(float z) { return max_nan(z, 0.0f); }
__device__ __forceinline__ float gelu(float z) {
  const float a = cut<NormalTail>(z);
  return fmaf(-a, tail<NormalTail>(a), relu(z));
}
__device__ __forceinline__ float gelu_tanh(float z) {
  const float a = cut<TanhTail>(z);
  return fmaf(-a, tail<TanhTail>(a), relu(z));
}
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }

// Slopes.  With m(a) = t(a) - a f(a), f the density, the slope is m for negative and 1 - m for positive arguments.
__device__ __forceinline__ float from_tail(float z, float m) { return z < 0.0f ? m : 1.0f - m; }
__device__ __forceinline__ float relu_slope(float z) { return z > 0.0f ? 1.0f : (z != z ? z : 0.0f); }
__device__ __forceinline__ float gelu_slope(float z) {
  const float a = cut<NormalTail>(z);
  return from_tail(z, fmaf(-a * INV_SQRT_2PI, ex2(-0.5f * LOG2E * a * a), tail<NormalTail>(a)));
}
__device__ __forceinline__ float gelu_tanh_slope(float z) {        // f = t (1 - t) 2 c (1 + 3 * 0.044715 a^2)
  const float a = cut<TanhTail>(z);
  const float t = tail<TanhTail>(a);
  return from_tail(z, fmaf(-a * t * (1.0f - t), 2.0f * GELU_C * fmaf(3.0f * GELU_A * a, a, 1.0f), t));
}
__device__ __forceinline__ float silu_slope(float z) {             // f = t (1 - t)
  const float a = min_nan(fabsf(z), 128.0f);
  const float t = sigmoid(-a);
  return from_tail(z, fmaf(-a * t, 1.0f - t, t));
}

// one activation, chosen at run time
__device__ __forceinline__ float value_of(int kind, float z) {
  switch (kind) {
    case BIMASK_ACT_RELU: return relu(z);
    case BIMASK_ACT_GELU: return gelu(z);
    case BIMASK_ACT_GELU_TANH: return gelu_tanh(z);
    case BIMASK_ACT_SILU: return silu(z);
    default: return z;
  }
}

// ---- the same on pairs ----
__device__ __forceinline__ Pair sigmoid2(Pair minus_log2e_x) {     // of -log2(e) x
  return map2(add2(map2(minus_log2e_x, [](float v) { return ex2(v); }), both(1.0f)), [](float v) { return rcp(v); });
}
__device__ __forceinline__ Pair relu2(Pair z) { return map2(z, [](float v) { return max_nan(v, 0.0f); }); }
template <typename T>
__device__ __forceinline__ Pair gelu2(Pair z) {
  const Pair a = map2(z, [](float v) { return cut<T>(v); });
  Pair p = both(T::c(T::N - 1));
#pragma unroll
  for (int i = T::N - 2; i >= 0; --i) p = fma2(p, a, both(T::c(i)));
  return fma2(map2(a, [](float v) { return -v; }), map2(p, [](float v) { return ex2(v); }), relu2(z));
}
__device__ __forceinline__ Pair silu2(Pair z) { return mul2(z, sigmoid2(mul2(z, both(-LOG2E)))); }

template <int KIND>
__device__ __forceinline__ Pair value2(Pair z) {
  return KIND == BIMASK_ACT_RELU ? relu2(z) : KIND == BIMASK_ACT_GELU ? gelu2<NormalTail>(z) : KIND == BIMASK_ACT_GELU_TANH ? gelu2<TanhTail>(z)
         : KIND == BIMASK_ACT_SILU ? silu2(z) : z;
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
constexpr float ROUNDER = 12582912.0f;                    // 1.5 * 2^23
__device__ __forceinline__ uint32_t round_bits(float x, float inv) { return __float_as_uint(fmaf(x, inv, ROUNDER)); }

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
