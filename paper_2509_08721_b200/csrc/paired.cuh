// Paired fp32 arithmetic of sm_100 (two floats an instruction), and a maximum that keeps NaN.
#pragma once

#include <cuda_runtime.h>

namespace sapo {

// (fma.rn.f32x2 and its kin, each half rounded like the scalar operation)
#define SAPO_F32X2(name, ptx)                                                                             \
  __device__ __forceinline__ float2 name(float2 a, float2 b) {                                            \
    float2 d;                                                                                             \
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t" ptx                 \
        " d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"                                                          \
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));                                 \
    return d;                                                                                             \
  }
SAPO_F32X2(add2, "add.rn.f32x2")
SAPO_F32X2(mul2, "mul.rn.f32x2")
#undef SAPO_F32X2
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
// the larger of two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

}  // namespace sapo
