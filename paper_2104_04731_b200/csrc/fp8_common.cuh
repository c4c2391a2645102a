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

// 16 consecutive elements from a 16-byte boundary.
__device__ __forceinline__ void load16(const float* p, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 f = *reinterpret_cast<const float4*>(p + 4 * i);
    v[4 * i] = f.x;
    v[4 * i + 1] = f.y;
    v[4 * i + 2] = f.z;
    v[4 * i + 3] = f.w;
  }
}
template <typename T>
__device__ __forceinline__ void load16(const T* p, float* v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 u = *reinterpret_cast<const uint4*>(p + 8 * i);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) unpack2<T>(w[j], &v[8 * i + 2 * j], &v[8 * i + 2 * j + 1]);
  }
}

// Block quantisation q = nearest 8-bit value of x * F / amax.  With amax = m * 2^e, 1 <= m < 2, the quotient is
// (x * F * 2^-e) / m: the first factor is exact for 16-bit x (F = 1.75 * 2^n adds two bits) and cannot overflow.
// A value that lies half way between two 8-bit values has to stay there (inputs of few bits meet such values
// often), so the division is rounded correctly: Markstein's theorem (P. Markstein, Computation of elementary
// functions on the IBM RISC System/6000 processor, IBM J. Res. Dev. 34, 1990) - with r the correctly rounded
// reciprocal of m, q0 = u * r, the residual u - q0 * m formed exactly by one FMA and q0 + residual * r is the
// correctly rounded quotient.  Four operations an element and one reciprocal a block.
struct BlockScale {
  float scale;  // amax / F
  float c;      // F * 2^-e
  float m, r;   // mantissa of amax and its reciprocal
};
template <int QT>
__device__ __forceinline__ BlockScale block_scale(float amax) {
  constexpr float F = QT == B2C_E4M3 ? 448.0f : 57344.0f;
  amax = fmaxf(amax, kMinAmax);
  BlockScale b;
  b.scale = __fdiv_rn(amax, F);
  const int bits = __float_as_int(amax);
  b.c = amax == INFINITY ? 0.0f : __int_as_float(__float_as_int(F) - (((bits >> 23) - 127) << 23));
  b.m = __int_as_float((bits & 0x7FFFFF) | 0x3F800000);
  b.r = __frcp_rn(b.m);
  return b;
}
__device__ __forceinline__ float scaled(const BlockScale& b, float x) {
  const float u = x * b.c;
  const float q0 = u * b.r;
  return fmaf(fmaf(-q0, b.m, u), b.r, q0);
}
// Two values, rounded to nearest even, saturating (a correctly rounded quotient is at most F anyway); NaN stays.
template <int QT>
__device__ __forceinline__ uint32_t cvt2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, QT == B2C_E4M3 ? __NV_E4M3 : __NV_E5M2);
}
template <int QT>
__device__ __forceinline__ uint4 quantize16(const BlockScale& b, const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = cvt2<QT>(scaled(b, v[4 * i]), scaled(b, v[4 * i + 1])) |
           (cvt2<QT>(scaled(b, v[4 * i + 2]), scaled(b, v[4 * i + 3])) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float fp8_to_float(uint8_t q, int type) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw(q, type == B2C_E4M3 ? __NV_E4M3 : __NV_E5M2);
  return __half2float(__half(h));
}

// (the quotient within two units of rounding instead of a half: five operations instead of some twenty, and 64 of them stand
// between the last MMA of a tile and the next one's; a denominator beyond 2^126 gives 0, as it should)
__device__ __forceinline__ float silu(float v) { return __fdividef(v, 1.0f + expf(-v)); }

}  // namespace
}  // namespace b2c
