// Arithmetic shared by the tensor-core kernels of the exact cross attention.
#pragma once

#include "tc_common.cuh"

namespace tcx {

// max of two and of three that hands NaNs on
__device__ __forceinline__ float max2n(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
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

// (a, b) = 2^(a, b) on the multiply-add pipe: as exp2_poly2 of tc_common.cuh, with the quartic that exp2_poly_fit.py's fit(4) gives
// (largest relative error 2.9e-6, 3.0e-6 with its sums in fp32): what a sum with one pair of eight from here is off by stays within
// fp32's own errors, which the cubic's 8.6e-5 does not.  Arguments below -125 give 2^-125.
// NANS: a NaN gives a NaN.  The bound below hands it on, and the power of two comes in by a product, which does too: added to the exponent's
// field it would make a finite number of it.
template <bool NANS>
__device__ __forceinline__ void exp2_quartic2(uint32_t& a, uint32_t& b) {
  const float x0 = NANS ? max2n(__uint_as_float(a), -125.f) : fmaxf(__uint_as_float(a), -125.f);
  const float x1 = NANS ? max2n(__uint_as_float(b), -125.f) : fmaxf(__uint_as_float(b), -125.f);
  uint32_t r0, r1, p0, p1;
  asm("{\n\t.reg .b64 x, r, n, f, p, c;\n\t"
      "mov.b64 x, {%4, %5};\n\t"
      "mov.b64 c, {0x4B400000, 0x4B400000};\n\t"          // 1.5 * 2^23
      "add.rm.f32x2 r, x, c;\n\t"
      "mov.b64 c, {0xCB400000, 0xCB400000};\n\t"
      "add.rn.f32x2 n, r, c;\n\t"                          // n = floor(x), exact
      "mov.b64 c, {0xBF800000, 0xBF800000};\n\t"
      "fma.rn.f32x2 f, n, c, x;\n\t"                       // f = x - n
      "mov.b64 c, {0x3C5BFB98, 0x3C5BFB98};\n\t"          // c4 = 0.01342668
      "mov.b64 p, {0x3D55FC34, 0x3D55FC34};\n\t"          // c3 = 0.05224247
      "fma.rn.f32x2 p, f, c, p;\n\t"
      "mov.b64 c, {0x3E771228, 0x3E771228};\n\t"          // c2 = 0.2412802
      "fma.rn.f32x2 p, p, f, c;\n\t"
      "mov.b64 c, {0x3F316B63, 0x3F316B63};\n\t"          // c1 = 0.69304484
      "fma.rn.f32x2 p, p, f, c;\n\t"
      "mov.b64 c, {0x3F800000, 0x3F800000};\n\t"
      "fma.rn.f32x2 p, p, f, c;\n\t"
      "mov.b64 {%0, %1}, r;\n\t"
      "mov.b64 {%2, %3}, p;\n\t}"
      : "=r"(r0), "=r"(r1), "=r"(p0), "=r"(p1)
      : "f"(x0), "f"(x1));
  if constexpr (NANS) {
    a = (r0 << 23) + 0x3f800000u;                      // 2^n: n in r's low bits
    b = (r1 << 23) + 0x3f800000u;
    asm("{\n\t.reg .b64 x, p;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 p, {%2, %3};\n\tmul.rn.f32x2 x, x, p;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+r"(a), "+r"(b)
        : "r"(p0), "r"(p1));
  } else {
    a = p0 + (r0 << 23);
    b = p1 + (r1 << 23);
  }
}

// The products' issue.  One elected lane issues; what it takes to say a product (two descriptors, two addresses) has to be a
// constant away from a value that the warp holds, or the issue of a tile's few short products takes longer than the products:
// the loop below is unrolled, with the steps that d has not (d < D) left out by a warp-uniform branch.
struct Desc {
  uint32_t lo, hi;
  __device__ __forceinline__ Desc(uint64_t d) : lo((uint32_t)d), hi((uint32_t)(d >> 32)) {}
};
// D [128 x N] = A [128 x 16 steps] B [N x 16 steps]^T, both K-major in panels of 64 columns of A_PANEL and B_PANEL bytes
template <int STEPS, uint32_t A_PANEL, uint32_t B_PANEL>
__device__ __forceinline__ void issue_rows(uint32_t d_tmem, Desc a, Desc b, uint32_t idesc, int steps) {
#pragma unroll
  for (int k = 0; k < STEPS; k++)
    if (k < steps)
      tc::mma_bf16_lh(d_tmem, a.lo + ((k >> 2) * A_PANEL + (k & 3) * 32) / 16, a.hi, b.lo + ((k >> 2) * B_PANEL + (k & 3) * 32) / 16, b.hi, idesc, k > 0);
}
// D [128 x N] (+)= A [128 x 16 STEPS] in tensor memory times B, whose 16 STEPS rows (of 128 bytes per panel) are the contraction
template <int STEPS>
__device__ __forceinline__ void issue_cols(uint32_t d_tmem, uint32_t a_tmem, Desc b, uint32_t idesc, uint32_t accumulate) {
#pragma unroll
  for (int k = 0; k < STEPS; k++) tc::mma_bf16_ta_lh(d_tmem, a_tmem + 8 * k, b.lo + k * (2048 / 16), b.hi, idesc, k > 0 ? 1u : accumulate);
}

// The same with A [128 x T] in two halves of T / 2 whose columns begin APART columns from each other
template <int T, int APART>
__device__ __forceinline__ void issue_halves(uint32_t d_tmem, uint32_t a_tmem, Desc b, uint32_t idesc, uint32_t accumulate) {
#pragma unroll
  for (int k = 0; k < T / 16; k++)
    tc::mma_bf16_ta_lh(d_tmem, a_tmem + k / (T / 32) * APART + k % (T / 32) * 8, b.lo + k * (2048 / 16), b.hi, idesc, k > 0 ? 1u : accumulate);
}

// 16 values of a row, all of its warp's lanes together: to fp32 sums of a piece, or rounded to the gradient.
__device__ __forceinline__ void store_row(bool on, const float (&x)[16], float* part, __nv_bfloat16* out) {
  if (on && part) {
#pragma unroll
    for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(part + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
  } else if (on) {
#pragma unroll
    for (int k = 0; k < 16; k += 8)
      *reinterpret_cast<uint4*>(out + k) = make_uint4(tc::pack_bf16(x[k], x[k + 1]), tc::pack_bf16(x[k + 2], x[k + 3]), tc::pack_bf16(x[k + 4], x[k + 5]), tc::pack_bf16(x[k + 6], x[k + 7]));
  }
  __syncwarp();
}
}  // namespace tcx
