// Arithmetic shared by the tensor-core kernels of the exact cross attention.
#pragma once

#include "tc_common.cuh"

namespace tcx {

// max of three that hands NaNs on
__device__ __forceinline__ float max3n(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void fma2(uint32_t& a, uint32_t& b, float m, float n) {      // (a, b) = (a, b) m + n
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+r"(a), "+r"(b)
      : "f"(m), "f"(n));
}

// (a, b) = (a, b) m + (n, o)
__device__ __forceinline__ void fma2v(uint32_t& a, uint32_t& b, float m, float n, float o) {
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %4};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+r"(a), "+r"(b)
      : "f"(m), "f"(n), "f"(o));
}
// (a, b) = ((a, b) + (n, o)) (p, q)
__device__ __forceinline__ void addmul2(uint32_t& a, uint32_t& b, float n, float o, uint32_t p, uint32_t q) {
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\t"
      "add.rn.f32x2 x, x, y;\n\tmul.rn.f32x2 x, x, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+r"(a), "+r"(b)
      : "f"(n), "f"(o), "r"(p), "r"(q));
}

}  // namespace tcx
