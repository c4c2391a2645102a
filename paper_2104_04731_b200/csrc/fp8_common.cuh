// Device code shared by the kernels of the 8-bit float operators: loads of the three wide types, the block
// quantisation arithmetic, conversions.  Included by each kernel translation unit; unnamed namespace.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "fp8_internal.h"

namespace b2c {

namespace {

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two fp32 values rounded to a packed pair (lo in the lower half).
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T>
__device__ __forceinline__ void unpack2(uint32_t w, float* lo, float* hi);
template <>
__device__ __forceinline__ void unpack2<__half>(uint32_t w, float* lo, float* hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  *lo = f.x;
  *hi = f.y;
}
template <>
__device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float* lo, float* hi) {
  *lo = __uint_as_float(w << 16);
  *hi = __uint_as_float(w & 0xFFFF0000u);
}

// A pair of fp32 values in one 64-bit register pair; two multiplications or FMAs are one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(f32x2 v, float* lo, float* hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(v)); }
__device__ __forceinline__ void fma2(f32x2* acc, f32x2 v, f32x2 f) { asm volatile("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(*acc) : "l"(v), "l"(f)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2_of(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// 16 consecutive elements from a 16-byte boundary, as they lie in memory, and widened.
template <typename T>
struct Raw16 {
  uint4 u[sizeof(T)];
};
template <typename T>
__device__ __forceinline__ Raw16<T> load_raw16(const T* p) {
  Raw16<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); ++i) r.u[i] = reinterpret_cast<const uint4*>(p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ void widen16(const Raw16<T>& r, float* v) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); ++i) {
    const uint32_t w[4] = {r.u[i].x, r.u[i].y, r.u[i].z, r.u[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) v[4 * i + j] = __uint_as_float(w[j]);
      else unpack2<T>(w[j], &v[8 * i + 2 * j], &v[8 * i + 2 * j + 1]);
    }
  }
}

// Largest magnitude of 16 elements, NaN left out; packed types two at a time.
__device__ __forceinline__ float raw_max(const Raw16<float>& r) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = fmaxf(m, fmaxf(fmaxf(fabsf(__uint_as_float(r.u[i].x)), fabsf(__uint_as_float(r.u[i].y))),
                       fmaxf(fabsf(__uint_as_float(r.u[i].z)), fabsf(__uint_as_float(r.u[i].w)))));
  return m;
}
template <typename T, typename T2>
__device__ __forceinline__ float raw_max2(const Raw16<T>& r) {
  T2 m[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w[4] = {r.u[i].x & 0x7FFF7FFFu, r.u[i].y & 0x7FFF7FFFu, r.u[i].z & 0x7FFF7FFFu, r.u[i].w & 0x7FFF7FFFu};
    const T2* p = reinterpret_cast<const T2*>(w);
    m[i] = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
  }
  const T2 both = __hmax2(m[0], m[1]);
  const float lo = to_float<T>(both.x), hi = to_float<T>(both.y);
  return fmaxf(fmaxf(lo, hi), 0.0f);  // (NaN where a half has nothing else: dropped here)
}
__device__ __forceinline__ float raw_max(const Raw16<__half>& r) { return raw_max2<__half, __half2>(r); }
__device__ __forceinline__ float raw_max(const Raw16<__nv_bfloat16>& r) { return raw_max2<__nv_bfloat16, __nv_bfloat162>(r); }

// Block quantisation q = nearest 8-bit value of x * F / amax.  With amax = m * 2^e, 1 <= m < 2, the quotient is
// (x * F * 2^-e) / m: the first factor is exact for 16-bit x (F = 1.75 * 2^n adds two bits) and cannot overflow.
// A value that lies half way between two 8-bit values has to stay there (inputs of few bits meet such values
// often), so the division is rounded correctly: Markstein's theorem (P. Markstein, Computation of elementary
// functions on the IBM RISC System/6000 processor, IBM J. Res. Dev. 34, 1990) - with r the correctly rounded
// reciprocal of m, q0 = u * r, the residual u - q0 * m formed exactly by one FMA and q0 + residual * r is the
// correctly rounded quotient.  Four operations an element, two elements an instruction, and one reciprocal a block.
struct BlockScale {
  float scale;       // amax / F
  f32x2 c, r, neg_m;  // F * 2^-e; reciprocal of m; -m: each twice, for two values at once
};
template <int QT>
__device__ __forceinline__ BlockScale block_scale(float amax) {
  constexpr float F = QT == B2C_E4M3 ? 448.0f : 57344.0f, R = 1.0f / F;
  amax = fmaxf(amax, kMinAmax);
  BlockScale b;
  // (the quotient by a constant the same way; an infinite amax would give NaN)
  const float q0 = amax * R;
  b.scale = amax == INFINITY ? INFINITY : fmaf(fmaf(-q0, F, amax), R, q0);
  const int bits = __float_as_int(amax);
  const float c = amax == INFINITY ? 0.0f : __int_as_float(__float_as_int(F) - (((bits >> 23) - 127) << 23));
  const float m = __int_as_float((bits & 0x7FFFFF) | 0x3F800000);
  const float r = __frcp_rn(m);
  b.c = pair_of(c, c);
  b.r = pair_of(r, r);
  b.neg_m = pair_of(-m, -m);
  return b;
}
// Two values, rounded to nearest even, saturating (a correctly rounded quotient is at most F anyway); NaN stays.
template <int QT>
__device__ __forceinline__ uint32_t quantize2(const BlockScale& b, float lo, float hi) {
  const f32x2 u = mul2(pair_of(lo, hi), b.c);
  const f32x2 q0 = mul2(u, b.r);
  const f32x2 q = fma2_of(fma2_of(q0, b.neg_m, u), b.r, q0);
  float2 f;
  unpair(q, &f.x, &f.y);
  return __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, QT == B2C_E4M3 ? __NV_E4M3 : __NV_E5M2);
}
template <int QT>
__device__ __forceinline__ uint4 quantize16(const BlockScale& b, const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __byte_perm(quantize2<QT>(b, v[4 * i], v[4 * i + 1]), quantize2<QT>(b, v[4 * i + 2], v[4 * i + 3]), 0x5410);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// silu(v) = v / (1 + e^-v), for negative v as v e^v / (1 + e^v): the divisor stays between one and two (1 + e^-v leaves the range of the
// quotient below v = -87, where v e^v has not left that of fp32).  The quotient within two units of rounding instead of a half: seven
// operations instead of some twenty, and 64 of them stand between the last MMA of a tile and the next one's.
__device__ __forceinline__ float silu(float v) {
  const float e = expf(-fabsf(v));
  return __fdividef(v < 0.0f ? v * e : v, 1.0f + e);
}

}  // namespace
}  // namespace b2c
