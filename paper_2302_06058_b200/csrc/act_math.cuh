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

// The activations, two values at a time.  Both GELUs are z times a distribution function F with F(-a) = 1 - F(a), so
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
__device__ __forceinline__ float cut(float z) { return min_nan(fabsf(z), T::CUT); }

// sigma(x) = 1 / (1 + e^-x), given -log2(e) x; e^-x = inf for very negative x gives 0
__device__ __forceinline__ Pair sigmoid2(Pair minus_log2e_x) {
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
// z is cut off at the least finite number: minus infinity times 0 would be NaN where the GELUs, and the limit, are 0
__device__ __forceinline__ Pair silu2(Pair z) {
  return mul2(map2(z, [](float v) { return max_nan(v, -3.402823466e38f); }), sigmoid2(mul2(z, both(-LOG2E))));
}

template <int KIND>
__device__ __forceinline__ Pair value2(Pair z) {
  return KIND == BIMASK_ACT_RELU ? relu2(z) : KIND == BIMASK_ACT_GELU ? gelu2<NormalTail>(z) : KIND == BIMASK_ACT_GELU_TANH ? gelu2<TanhTail>(z)
         : KIND == BIMASK_ACT_SILU ? silu2(z) : z;
}

// the same, the activation chosen at run time, once for the whole array
template <int KIND, int N>
__device__ __forceinline__ void apply_one(Pair (&z)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) z[i] = value2<KIND>(z[i]);
}
template <int N>
__device__ __forceinline__ void apply(int kind, Pair (&z)[N]) {
  switch (kind) {
    case BIMASK_ACT_RELU: apply_one<BIMASK_ACT_RELU>(z); break;
    case BIMASK_ACT_GELU: apply_one<BIMASK_ACT_GELU>(z); break;
    case BIMASK_ACT_GELU_TANH: apply_one<BIMASK_ACT_GELU_TANH>(z); break;
    case BIMASK_ACT_SILU: apply_one<BIMASK_ACT_SILU>(z); break;
    default: break;
  }
}
// Slopes.  With m(a) = t(a) - a f(a), f the density, the slope is m(a) for negative and 1 - m(a) for positive arguments:
// 1/2 + (1/2 - m(a)) with the sign of z.  For the GELUs m(a) = e^(-a^2/2) P(a): m over the normal density is smooth and P is
// the minimax fit of m, by linear programming; errors in fp32 3.1e-7 (degree 9) and 1.5e-7 (tanh form, degree 10).
struct NormalSlope {
  static constexpr int N = 10;
  static __device__ __forceinline__ constexpr float c(int i) {
    constexpr float k[N] = {0.499999743f, -0.797864899f, 0.249752293f, -0.131772884f, 0.0594967943f, -0.0222308766f, 0.00638280561f,
                            -0.00127116217f, 0.000151941892f, -8.06307163e-06f};
    return k[i];
  }
};
struct TanhSlope {
  static constexpr int N = 11;
  static __device__ __forceinline__ constexpr float c(int i) {
    constexpr float k[N] = {0.499999899f, -0.797877544f, 0.249918295f, -0.131275385f, 0.0614912298f, -0.0257054393f, 0.00879214436f,
                            -0.00278788268f, 0.000777319758f, -0.000125037125f, 7.79687128e-06f};
    return k[i];
  }
};
__device__ __forceinline__ Pair signed_half(Pair z, Pair half_minus_m) {    // 1/2 + the second, given the signs of the first
  float x, y, a, b;
  split(z, x, y);
  split(half_minus_m, a, b);
  return add2(pair(__uint_as_float(__float_as_uint(a) ^ (__float_as_uint(x) & 0x80000000u)),
                   __uint_as_float(__float_as_uint(b) ^ (__float_as_uint(y) & 0x80000000u))), both(0.5f));
}
template <typename S>
__device__ __forceinline__ Pair gelu_slope2(Pair z) {
  const Pair a = map2(z, [](float v) { return cut<NormalTail>(v); });       // the exponential is 0 in fp32 from there on
  const Pair g = map2(mul2(mul2(a, both(-0.5f * LOG2E)), a), [](float v) { return ex2(v); });
  Pair p = both(-S::c(S::N - 1));
#pragma unroll
  for (int i = S::N - 2; i >= 0; --i) p = fma2(p, a, both(-S::c(i)));
  return signed_half(z, fma2(p, g, both(0.5f)));
}
__device__ __forceinline__ Pair silu_slope2(Pair z) {                       // t = sigma(-a), f = t (1 - t)
  const Pair a = map2(z, [](float v) { return min_nan(fabsf(v), 128.0f); });
  const Pair t = sigmoid2(mul2(a, both(LOG2E)));
  const Pair f = fma2(mul2(t, both(-1.0f)), t, t);
  return signed_half(z, add2(fma2(a, f, both(0.5f)), mul2(t, both(-1.0f))));
}
__device__ __forceinline__ Pair relu_slope2(Pair z) { return map2(z, [](float v) { return v > 0.0f ? 1.0f : (v != v ? v : 0.0f); }); }

template <int KIND>
__device__ __forceinline__ Pair slope2(Pair z) {
  return KIND == BIMASK_ACT_RELU ? relu_slope2(z) : KIND == BIMASK_ACT_GELU ? gelu_slope2<NormalSlope>(z)
         : KIND == BIMASK_ACT_GELU_TANH ? gelu_slope2<TanhSlope>(z) : silu_slope2(z);
}

}  // namespace act

// ---- 8-bit checkpoint ---------------------------------------------------------------------------
namespace ckpt {

// The scale depends on max |x| only through the comparison with 127 * 2^e, whose mantissa ends within the seven bits of
// a bf16: so the maximum may be taken on |x| rounded UP to bf16, 16 bits that compare as integers (NaN above infinity
// above every finite value).
__device__ __forceinline__ uint32_t up16(float abs_x) { return (__float_as_uint(abs_x) + 0xFFFFu) >> 16; }

// Scale byte of a block from that maximum h: 2^(s-127) is the smallest power of two, not below 2^-126, with
// max |x| <= 127 * 2^(s-127); 255: the block holds a NaN or a magnitude above 127 * 2^121 (bf16 0x7F7E), whose byte would be
// 64 steps of 2^122 and stand for 2^128, infinity.
constexpr uint32_t LARGEST = 0x7F7Eu;
__device__ __forceinline__ uint32_t scale_of(uint32_t h) {
  const int s = (int)((h + 1u) >> 7) - 6;                 // exponent of h, one more when its mantissa is above 1.984375 = 127 / 64
  return h > LARGEST ? 255u : (uint32_t)(s < 1 ? 1 : s);
}
// 2^(127 - s): x times it is exact, and rounds to the byte
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127); NaN for 255
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s == 255u ? 0x7FC00000u : s << 23); }

// Round x / 2^(s-127) to the nearest integer (ties to even): it is the low byte of the result's bits.
constexpr float ROUNDER = 12582912.0f;                    // 1.5 * 2^23
__device__ __forceinline__ uint32_t round_bits(float x, float inv) { return __float_as_uint(fmaf(x, inv, ROUNDER)); }

// bytes 0..3 of w times the scale, as two pairs.  The byte plus 128 goes into the low bits of 2^23: exact.
__device__ __forceinline__ void decode4(uint32_t w, act::Pair scale, act::Pair* out) {
  const uint32_t u = w ^ 0x80808080u;
  const act::Pair bias = act::both(-8388736.0f);          // -(2^23 + 128)
  out[0] = act::mul2(act::add2(act::pair(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7540)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7541))), bias), scale);
  out[1] = act::mul2(act::add2(act::pair(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7542)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7543))), bias), scale);
}

}  // namespace ckpt

__device__ __forceinline__ uint32_t pack_bf16_f(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_bf16_p(act::Pair v) {
  float lo, hi;
  act::split(v, lo, hi);
  return pack_bf16_f(lo, hi);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ act::Pair bf16_pair(uint32_t w) { return act::pair(bf16_lo(w), bf16_hi(w)); }

}  // namespace bimask
