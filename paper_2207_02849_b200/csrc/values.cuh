// Values of the operators' three types: conversions, and pairs of fp32 values.
#pragma once
#include "common.cuh"

namespace betty {

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

// two neighbouring values into one 32-bit word, one conversion instruction
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&v;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *(const uint32_t*)&v;
}
template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float& a, float& b) {
  const float2 v = __half22float2(*(const __half2*)&w);
  a = v.x; b = v.y;
}

// row `row` of a matrix with rows of `ld_bytes` bytes (both below 2^32: one wide multiply)
template <typename T>
__device__ __forceinline__ const T* row_at(const void* base, int64_t row, uint32_t ld_bytes) {
  return (const T*)((const char*)base + (uint64_t)(uint32_t)row * ld_bytes);
}
template <typename T>
__device__ __forceinline__ T* row_at(void* base, int64_t row, uint32_t ld_bytes) {
  return (T*)((char*)base + (uint64_t)(uint32_t)row * ld_bytes);
}

__device__ __forceinline__ float reciprocal(float v) {        // 1 ulp; 0 for an overflowed power
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float exp2_f(float v) {            // within 2^-22 of itself
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float between(float v, float low, float high) {        // NaN stays
  float r;
  asm("{\n\t.reg .f32 a;\n\tmax.NaN.f32 a, %1, %2;\n\tmin.NaN.f32 %0, a, %3;\n\t}" : "=f"(r) : "f"(v), "f"(low), "f"(high));
  return r;
}
// s = 1 / (1 + e^-v) and n = 1 - s, each within 7e-7 of itself, for results in fp32.  The power of two is taken of the rounded product
// with log2 e, and what that lacks of -v (2^-24 of it, which alone would be |v| 2^-24 of the power) is made good as a factor.
// From -87.3 down s is below the normal numbers and 0; the bounds keep e finite and an infinite v from leaving a NaN.
__device__ __forceinline__ void sigmoid_parts(float v, float& s, float& n) {
  const float a = between(v, -88.7f, 104.f), p = a * -1.4426950408889634f;
  const float lack = fmaf(p, 1.9046542e-9f, fmaf(p, -0.693147182f, -a));        // -a - p ln 2, ln 2 in two parts
  const float e0 = exp2_f(p), e = fmaf(e0, lack, e0);
  s = reciprocal(1.f + e);
  n = v < 0.f ? 1.f - s : e * s;
}

// ---- pairs of fp32 values: one instruction for two products or sums ----
struct alignas(8) f2 { float x, y; };
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ f2 both(float v) { return f2{v, v}; }
__device__ __forceinline__ void pairs(f2 (&o)[4], const float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = f2{v[2 * k], v[2 * k + 1]};
}
__device__ __forceinline__ void singles(float (&o)[8], const f2 (&v)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) { o[2 * k] = v[k].x; o[2 * k + 1] = v[k].y; }
}

}  // namespace betty
