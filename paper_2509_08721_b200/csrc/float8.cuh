// 8-bit floating point (e4m3: 4 bits of exponent, 3 of fraction, largest value 448) with one fp32 scale per group of 128.
#pragma once

#include <cuda_fp8.h>
#include <stdint.h>

namespace sapo {

constexpr int F8_GROUP = 128;
constexpr float F8_TOP = 448.f;
constexpr float F8_TINY = 1.504632769052528e-36f;   // 2^-119: below it 448 (1/a) leaves the fp32 range; such a group is stored as zeros

// scale of a group with largest magnitude a, and the factor that takes its values to [-448, 448] (a NaN or infinite: NaN, 0)
__device__ __forceinline__ void f8_group(float a, float& scale, float& inv) {
  const bool finite = a < __int_as_float(0x7f800000);
  scale = !finite ? __int_as_float(0x7fffffff) : (a >= F8_TINY ? __fmul_rn(a, 1.f / F8_TOP) : 0.f);
  inv = finite && a >= F8_TINY ? __fmul_rn(F8_TOP, __frcp_rn(a)) : 0.f;
}
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
__device__ __forceinline__ void f8_unpack4(uint32_t q, float (&v)[4]) {
  const __half2 lo = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q & 0xFFFFu), __NV_E4M3));
  const __half2 hi = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> 16), __NV_E4M3));
  const float2 a = __half22float2(lo), b = __half22float2(hi);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

}  // namespace sapo
