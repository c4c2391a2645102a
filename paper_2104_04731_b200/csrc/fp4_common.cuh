// Device code shared by the kernels of the 4-bit float operators: scales of blocks, conversion to 4 bits and back.  Included by each kernel
// translation unit; unnamed namespace.
#pragma once

#include "fp4_internal.h"
#include "fp8_common.cuh"

namespace b2c {

namespace {

constexpr uint32_t kInfBits = 0x7F800000u;

// The tensor's factor, and what is formed of it once a thread.
struct Factor4 {
  float g;
  bool few_bits;             // 17 at most: scale * g is exact in fp32, and so are its products with the borders between 4-bit values
  float six, six_lo, inv_6;  // 6 g as the sum of two, and its reciprocal
};
__device__ __forceinline__ Factor4 load_factor4(const float* p, int format) {
  Factor4 f;
  f.g = p != nullptr && format == B2C_NVFP4 ? fminf(fmaxf(*p, 0x1p-100f), 0x1p100f) : 1.0f;
  f.few_bits = (__float_as_uint(f.g) & 0x7Fu) == 0;
  f.six = 6.0f * f.g;
  f.six_lo = fmaf(6.0f, f.g, -f.six);  // (26 bits in all: exact)
  f.inv_6 = __frcp_rn(f.six);
  return f;
}

// A number on the same side as the quotient x / (hi + lo) of every border with few bits: t, which is the quotient q (good to some units) rounded to
// as many bits as a border has, moved by 2^-10 of itself (less than to the next such number) to where d = x - t * (hi + lo) says.
// x - t * hi is exact where it is small, and the rounding of the last sum keeps its sign.  Where d is not 0 it is 2^-36 of the divisor at least (the
// lowest border between scales is 2^-10, and 6 g has 26 bits), and `large` makes it more than 1/2.  Below divisors of 2^-87 `large` is at its limit:
// d is a multiple of 2^-134 (of the last places of g, 2^-123, of a scale, 2^-9, and of a border, 2^-2), so 2^-7 are left and t moves by 2^-16 of
// itself, still to the right side.  All of it on the unit of the multiplications, which has twice the rate of that of comparisons.
__device__ __forceinline__ float side_of(float t, float d, float large) {
  return fmaf(fabsf(t), fmaf(__saturatef(fmaf(d, large, 0.5f)), 0x1p-9f, -0x1p-10f), t);
}
__device__ __forceinline__ float large_of(float inverse) { return fminf(inverse * 0x1p40f, 0x1p127f); }

// Scale of a block.  amax: bits of its largest magnitude (as whole numbers these are ordered as the magnitudes, and NaN is the largest).
struct Scale4 {
  uint32_t code;   // as stored
  float r;         // reciprocal of the step, 0 where the values are zeros
  float step, lo;  // NV: the step is their sum, lo is 0 under a factor of few bits
};
// MX: with amax = m * 2^k, 1 <= m < 2, the least power of two s with amax <= 6 s = 1.5 * 2^2 s is 2^(k - 2), or twice that for m > 1.5.
__device__ __forceinline__ Scale4 scale_mx(uint32_t amax) {
  Scale4 s;
  const int e = (int)((amax + 0x3FFFFFu) >> 23) - 2;  // biased; the addend carries from m > 1.5 on
  const uint32_t code = (uint32_t)max(e, 0);
  const bool fine = amax < kInfBits;
  s.code = fine ? code : 255u;
  s.r = fine ? __uint_as_float((254u - code) << 23) : 0.0f;  // 2^(127 - code), a power of two: products with it are exact
  s.step = s.lo = 0.0f;
  return s;
}
// NV: the E4M3 value nearest to the real quotient amax / (6 g).  A border between two E4M3 values has 5 bits (t is rounded to them by Veltkamp's
// sum: T. J. Dekker, A floating-point technique for extending the available precision, Numer. Math. 18, 1971), so its product with 6 g has 31 at
// most, and amax is that product or differs from it by 2^-31 or more of itself.
__device__ __forceinline__ Scale4 scale_nv(uint32_t amax, const Factor4& f) {
  Scale4 s;
  const float a = __uint_as_float(amax), p = fminf(a * f.inv_6, 512.0f);
  const float c = __fmul_rn(p, 524289.0f), t = __fsub_rn(c, __fsub_rn(c, p));
  const float v = side_of(t, fmaf(-t, f.six_lo, fmaf(-t, f.six, a)), large_of(f.inv_6));
  const bool fine = amax < kInfBits;
  s.code = fine ? (uint32_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3) : 0x7Fu;
  const float e = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)s.code, __NV_E4M3)));
  s.step = e * f.g;
  s.lo = fmaf(e, f.g, -s.step);  // (28 bits in all: exact)
  float r;
  if (f.few_bits) r = __frcp_rn(s.step);
  else asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s.step));
  s.r = fine && s.code != 0 ? r : 0.0f;
  return s;
}
__device__ __forceinline__ float scale_value(uint32_t code, int format) {
  if (format == B2C_MXFP4) return code == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(code == 0 ? 0x400000u : code << 23);
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}

// Eight values to 4 bits each, to nearest even, saturating.
__device__ __forceinline__ uint32_t cvt_e2m1x8(const float* v) {
  uint32_t r;
  asm("{\n.reg .b8 b0, b1, b2, b3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
      "mov.b32 %0, {b0, b1, b2, b3};\n}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// Four values, in the lower half.
__device__ __forceinline__ uint32_t cvt_e2m1x4(const float* v) {
  uint32_t r;
  asm("{\n.reg .b8 b0, b1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      "mov.b32 %0, {b0, b1, b0, b1};\n}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
  return r & 0xFFFFu;
}
// Eight 4-bit values in halves, exact.
__device__ __forceinline__ void cvt_f16x8(uint32_t q, uint32_t* h) {
  asm("{\n.reg .b8 b0, b1, b2, b3;\n"
      "mov.b32 {b0, b1, b2, b3}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(q));
}

// N (8 or 16) values of one block to 4 bits each, as if x / (scale * g) had been rounded as a real number.
//   MX: multiplication by a power of two.
//   NV, few_bits: the correctly rounded quotient by Markstein's residual step (as in quantize2 of the 8-bit operators).  Every product of the step with a border t has 24
// bits at most, so x is either that product, and the quotient t itself, or differs from it by a unit of x's last place, more than half a
// unit of t's: the rounded quotient is on the same side.
//   NV else: by side_of, with four bits.  (Factors that come from a largest value of few bits put one number in 200 within 2^-23 of a border:
// deciding these by comparisons in 64 bits made 16384 x 8192 take 217 us.)
//   A block whose scale is the largest one may be beyond it by any factor: eight steps round to the same value, and stay finite.
template <int N>
__device__ __forceinline__ void quantise4(const Scale4& s, const Factor4& f, int format, const float* in, uint32_t* q) {
  float v[N], x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = in[i];
  if (format == B2C_NVFP4 && s.code == 0x7Eu) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fminf(fmaxf(x[i], -8.0f * s.step), 8.0f * s.step);
  }
  const f32x2 r = pair_of(s.r, s.r), neg = pair_of(-s.step, -s.step);
  if (format == B2C_MXFP4) {
#pragma unroll
    for (int i = 0; i < N; i += 2) unpair(mul2(pair_of(x[i], x[i + 1]), r), &v[i], &v[i + 1]);
  } else if (f.few_bits) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const f32x2 u = pair_of(x[i], x[i + 1]), q0 = mul2(u, r);
      unpair(fma2_of(fma2_of(q0, neg, u), r, q0), &v[i], &v[i + 1]);
    }
  } else {
    const f32x2 neg_lo = pair_of(-s.lo, -s.lo), split = pair_of(1048577.0f, 1048577.0f), zero = pair_of(0.0f, 0.0f);
    const float large = large_of(s.r);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      // (products as sums with 0: ptxas joins a packed product and the difference behind it to one operation, although both say .rn)
      const f32x2 u = pair_of(x[i], x[i + 1]), q0 = fma2_of(u, r, zero), c = fma2_of(q0, split, zero), t = sub2(c, sub2(c, q0));
      float tt[2], d[2];
      unpair(t, &tt[0], &tt[1]);
      unpair(fma2_of(t, neg_lo, fma2_of(t, neg, u)), &d[0], &d[1]);
#pragma unroll
      for (int j = 0; j < 2; ++j) v[i + j] = side_of(tt[j], d[j], large);
    }
  }
#pragma unroll
  for (int i = 0; i < N / 8; ++i) q[i] = cvt_e2m1x8(v + 8 * i);
  if (s.r == 0.0f) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) q[i] = 0;
  }
}
__device__ __forceinline__ Scale4 scale_of(uint32_t amax, const Factor4& f, int format) {
  return format == B2C_MXFP4 ? scale_mx(amax) : scale_nv(amax, f);
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The hidden rows of an expert layer are quantised from values that are off by the errors of their sums, so the residuals that decide
// borders exactly have nothing to decide: scale and quotients are formed in fp32.  A border moves by 3 units of 2^-24 at most: that of a scale by the
// roundings of 6 g, its reciprocal and the product, that of a value by those of the step, its reciprocal and the product.  (The step's reciprocal
// as 6 / (6 g) by a quick quotient was off by up to 8: values 3.7 units from a border went to the wrong side of it.)
struct QuickFactor4 {
  float g, inv_6;
};
__device__ __forceinline__ QuickFactor4 quick_factor4(const float* p, int format) {
  if (p == nullptr || format != B2C_NVFP4) return {1.0f, 1.0f / 6.0f};
  const float g = fminf(fmaxf(*p, 0x1p-100f), 0x1p100f);
  return {g, __frcp_rn(6.0f * g)};
}
__device__ __forceinline__ Scale4 quick_scale(uint32_t amax, const QuickFactor4& f, int format) {
  if (format == B2C_MXFP4) return scale_mx(amax);
  Scale4 s;
  const bool fine = amax < kInfBits;
  s.code = fine ? (uint32_t)__nv_cvt_float_to_fp8(__uint_as_float(amax) * f.inv_6, __NV_SATFINITE, __NV_E4M3) : 0x7Fu;
  const float t = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)s.code, __NV_E4M3)));
  s.r = fine && s.code != 0 ? __frcp_rn(t * f.g) : 0.0f;  // (the step is 2^-109 to 2^109)
  s.step = s.lo = 0.0f;
  return s;
}
template <int N>
__device__ __forceinline__ void quick_quantise4(const Scale4& s, const float* x, uint32_t* q) {
  float v[N];
  const f32x2 r = pair_of(s.r, s.r);
#pragma unroll
  for (int i = 0; i < N; i += 2) unpair(mul2(pair_of(x[i], x[i + 1]), r), &v[i], &v[i + 1]);
#pragma unroll
  for (int i = 0; i < N / 8; ++i) q[i] = cvt_e2m1x8(v + 8 * i);
  if constexpr (N == 4) q[0] = cvt_e2m1x4(v);
  if (s.r == 0.0f) {
#pragma unroll
    for (int i = 0; i < (N + 7) / 8; ++i) q[i] = 0;
  }
}
// The largest magnitude of three; NaN if one is.
__device__ __forceinline__ float max_abs3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// silu(gate) * up, silu as in the 8-bit layer with e^-|v| as a power of two whose exponent is one rounded product: the power is off by 1.25 |v| 2^-24 of
// itself more, and silu with it where v is negative; where it is positive by 1.25 v e^-v 2^-24, half a unit at most.
//   Below v = kFarGate (e^v is above 2^-122 there, and no longer counts beside 1) the power is formed 2^96 times too large and h is scaled back behind
// the product with up, which may be large: scales go down to 2^-127, and e^v alone leaves the range of fp32 at -87.  The range of the larger power
// ends at v = -153, below which h is 0.  The exponent is a sum rounded once, by less than without the shift.
//   Eight operations, two of them on the unit of 16 results a cycle, and four more with FAR, for gates that may be below kFarGate.
constexpr float kFarGate = -84.0f;
template <bool FAR>
__device__ __forceinline__ float quick_gated(float gate, float up) {
  const bool far = FAR && gate < kFarGate;
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(fabsf(gate), -1.44269504f, far ? 96.0f : 0.0f)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  const float h = (gate < 0.0f ? gate * e : gate) * r * up;
  return far ? h * 0x1p-96f : h;
}
// The least of three (a NaN is left out).
__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

}  // namespace
}  // namespace b2c
