// Position rotation and latent normalisation of bf16 rows, as the fused cache
// writer and the query rotation apply them.
//
// The writer's results are RN_bf16(RN_f32(exact)): the arithmetic carries the rounding
// errors of its fp32 operations along (error-free transformations: T. J. Dekker,
// Numer. Math. 18, 1971; D. E. Knuth, TAOCP 2, 4.2.2), which leaves about 2^-46
// relative (of rows near the ends of fp32's range too, which far_row tells apart). A
// plain fp32 evaluation is off by up to some 2^-22, which moves one
// bf16 value in about 2^13 and with it, now and then, the 2- or 4-bit code or the
// scale of a whole group; this way the cache holds the same bytes whatever order
// the sums are taken in. Queries, which nothing quantises, are rotated in plain fp32.
#pragma once
#include <cstdint>

#include "ptx.cuh"

namespace qmla {

// A value hi + lo with hi = RN_f32(value).
struct F2 {
  float hi, lo;
};
__device__ __forceinline__ F2 two_sum(float a, float b) {
  const float s = __fadd_rn(a, b);
  const float t = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ F2 two_prod(float a, float b) {
  const float p = __fmul_rn(a, b);
  return {p, __fmaf_rn(a, b, -p)};
}
__device__ __forceinline__ F2 add_f2(F2 a, F2 b) {
  const F2 s = two_sum(a.hi, b.hi);
  const float lo = __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo));
  const float hi = __fadd_rn(s.hi, lo);
  return {hi, __fsub_rn(lo, __fsub_rn(hi, s.hi))};
}

// The same for two values at once (the packed operations round like the others).
struct F2x2 {
  uint64_t hi, lo;
};
__device__ __forceinline__ uint64_t sub2(uint64_t a, uint64_t b) {
  return fma2(b, f32x2(-1.0f, -1.0f), a);
}
__device__ __forceinline__ F2x2 two_sum2(uint64_t a, uint64_t b) {
  const uint64_t s = add2(a, b), t = sub2(s, a);
  return {s, add2(sub2(a, sub2(s, t)), sub2(b, t))};
}

// RN_f32(a c + b s). Of an infinity, and past the largest float, the errors are NaN; the
// leading sum is then the result.
__device__ __forceinline__ float rotate1(float a, float c, float b, float s) {
  const F2 p = two_prod(a, c), q = two_prod(b, s);
  const F2 d = two_sum(p.hi, q.hi);
  const float r = __fadd_rn(d.hi, __fadd_rn(d.lo, __fadd_rn(p.lo, q.lo)));
  return fabsf(d.hi) <= 3.402823466e38f ? r : d.hi;
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight lanes hold one row of 64 channels, lane `piece` the channels 8 piece ..
// 8 piece + 7 in w. t is the row's entry of the angle table (cos[32] | sin[32]).
// All 32 lanes of the warp take part (t may be null in lanes without a row).
//   half-split (interleaved = false): channel i < 32 turns with channel i + 32,
//     which is four lanes away: x c - x' s below, x c + x' s above;
//   interleaved: channels 2 i and 2 i + 1 turn together.
struct Angles {
  float c[8], s[8];  // half-split: eight of each; interleaved: the first four
};
__device__ __forceinline__ void load_angles(Angles& a, const float* t, int piece, bool interleaved) {
  const float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float4* q = reinterpret_cast<const float4*>(t) + (interleaved ? piece : 2 * (piece & 3));
  const bool on = t != nullptr;
  const float4 c0 = on ? q[0] : z, s0 = on ? q[8] : z;
  const float4 c1 = on && !interleaved ? q[1] : z, s1 = on && !interleaved ? q[9] : z;
  a.c[0] = c0.x, a.c[1] = c0.y, a.c[2] = c0.z, a.c[3] = c0.w, a.c[4] = c1.x, a.c[5] = c1.y, a.c[6] = c1.z, a.c[7] = c1.w;
  a.s[0] = s0.x, a.s[1] = s0.y, a.s[2] = s0.z, a.s[3] = s0.w, a.s[4] = s1.x, a.s[5] = s1.y, a.s[6] = s1.z, a.s[7] = s1.w;
}
// EXACT: RN_bf16(RN_f32(exact)), else one fp32 product and one FMA.
template <bool EXACT>
__device__ __forceinline__ float rotate_value(float a, float c, float b, float s) {
  if constexpr (EXACT) return rotate1(a, c, b, s);
  return __fmaf_rn(a, c, __fmul_rn(b, s));
}
template <bool EXACT>
__device__ __forceinline__ void rotate_row(uint32_t (&w)[4], const Angles& a, int piece, bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = bf16_low(w[e]), y = bf16_high(w[e]);
      w[e] = pack_bf16(rotate_value<EXACT>(x, a.c[e], y, -a.s[e]), rotate_value<EXACT>(x, a.s[e], y, a.c[e]));
    }
  } else {
    const float sign = piece < 4 ? -1.0f : 1.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t o = __shfl_xor_sync(0xffffffffu, w[e], 4);
      w[e] = pack_bf16(rotate_value<EXACT>(bf16_low(w[e]), a.c[2 * e], bf16_low(o), sign * a.s[2 * e]),
                       rotate_value<EXACT>(bf16_high(w[e]), a.c[2 * e + 1], bf16_high(o), sign * a.s[2 * e + 1]));
    }
  }
}

// Adds the squares of eight bf16 values (each exact in fp32), even and odd channels
// side by side.
__device__ __forceinline__ void add_squares8(F2x2& sum, const uint32_t (&w)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t x = f32x2(bf16_low(w[e]), bf16_high(w[e]));
    const F2x2 t = two_sum2(sum.hi, mul2(x, x));
    sum = {t.hi, add2(sum.lo, t.lo)};
  }
}
__device__ __forceinline__ F2 square_sum8(const uint32_t (&w)[4]) {
  F2x2 sum = {0, 0};  // (pairs of zeros)
  add_squares8(sum, w);
  return add_f2({lo2(sum.hi), lo2(sum.lo)}, {hi2(sum.hi), hi2(sum.lo)});
}

// 1 / sqrt(sum / 512 + eps), by one Newton step from an fp32 estimate whose
// residual 1 - m y^2 is taken exactly.
__device__ __forceinline__ F2 row_rstd(F2 sum, float eps) {
  const F2 m = add_f2({__fmul_rn(sum.hi, 1.0f / 512.0f), __fmul_rn(sum.lo, 1.0f / 512.0f)}, {eps, 0.0f});
  const float y = __frsqrt_rn(m.hi);
  const F2 t = two_prod(y, y);
  const F2 p = two_prod(m.hi, t.hi);
  const float low = __fmaf_rn(m.lo, t.hi, __fmaf_rn(m.hi, t.lo, p.lo));
  const float r = __fsub_rn(__fsub_rn(1.0f, p.hi), low);
  return {y, __fmul_rn(0.5f, __fmul_rn(y, r))};
}

// Squares of fp32 leave its range long before the values do, and the errors that the sums
// carry along leave it sooner still: that arithmetic holds where the mean square plus eps
// lies within 2^-90 .. 2^90 (a square that underflows is then off by 2^-150, a residual
// of y^2 lies above 2^-138). Any other row (`far`; a NaN or an infinite sum too) is first
// multiplied by the power of two that brings the larger of its largest value and sqrt(eps)
// to about 1: x / sqrt(mean + eps) is the same for (f x, f^2 eps).
__device__ __forceinline__ bool far_row(F2 sum, float eps) {
  const float m = __fmaf_rn(sum.hi, 1.0f / 512.0f, eps);
  return !(m >= 0x1p-90f && m <= 0x1p90f);
}
// The largest of eight magnitudes, as the bits of a bf16 (above 0x7F80: a NaN).
__device__ __forceinline__ uint32_t largest8(const uint32_t (&w)[4]) {
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) v = __vmaxu2(v, w[e] & 0x7FFF7FFFu);
  return max(v & 0xFFFFu, v >> 16);
}
// f of a row whose largest magnitude is `top`. Its exponent stays within a float's normal
// range; what then lies above 1 or below it does so by a factor of 2^7 at most.
__device__ __forceinline__ float far_factor(uint32_t top, float eps) {
  int k = static_cast<int>(top >> 7) - 127;
  if (eps > 0.0f) k = max(k, (static_cast<int>(__float_as_uint(eps) >> 23) - 126) >> 1);
  return __uint_as_float(static_cast<uint32_t>(127 - max(-126, min(126, k))) << 23);
}
// Eight values times f: exact in bf16, but for what falls below 2^-126 of a row scaled down.
__device__ __forceinline__ void scale_words(uint32_t (&w)[4], float f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16(__fmul_rn(bf16_low(w[e]), f), __fmul_rn(bf16_high(w[e]), f));
}
// row_rstd of a row that has been scaled; with an infinite value 0 (x / inf), with a NaN NaN.
__device__ __forceinline__ F2 far_rstd(F2 sum, float eps, float f, uint32_t top) {
  const F2 r = row_rstd(sum, __fmul_rn(__fmul_rn(eps, f), f));
  if (top < 0x7F80u) return r;
  const float v = top == 0x7F80u ? 0.0f : __uint_as_float(0x7FC00000u);
  return {v, v};
}

// RN_bf16(RN_f32(x g rstd)) of eight values in place (x g is exact in fp32).
__device__ __forceinline__ void scale_row(uint32_t (&w)[4], const uint64_t (&g)[4], F2 rstd) {
  const uint64_t hi = f32x2(rstd.hi, rstd.hi), minus_hi = f32x2(-rstd.hi, -rstd.hi), minus_lo = f32x2(-rstd.lo, -rstd.lo);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t v = mul2(f32x2(bf16_low(w[e]), bf16_high(w[e])), g[e]);
    const uint64_t p = mul2(v, hi);
    // p less its rounding error less v lo
    const uint64_t y = sub2(p, fma2(v, minus_lo, fma2(v, minus_hi, p)));
    w[e] = pack_bf16(lo2(y), hi2(y));
  }
}

}  // namespace qmla
