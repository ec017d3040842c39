// float32 values as pairs of float16 limbs (x = hi + lo), the scales they are held at, and the panels they are stored in.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace {

constexpr uint32_t kPanel = 16384;                         // 128 rows x 64 float16
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
constexpr float kXScale = 16384.0f;                        // |X| <= 2 on entry and by the bound on the coefficients
constexpr float kAScale = 8192.0f;                         // |A| <= 4
// two float32 values at a time
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// x, y -> packed high limbs and packed low limbs (x - hi in one mixed-precision operation per value)
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
  hi = pack_f16(x, y);
  float a, b;
  asm("{\n\t.reg .b16 h0, h1, minus_one;\n\tmov.b32 {h0, h1}, %2;\n\tmov.b16 minus_one, 0xBC00;\n\t"
      "fma.rn.f32.f16 %0, h0, minus_one, %3;\n\tfma.rn.f32.f16 %1, h1, minus_one, %4;\n\t}"
      : "=f"(a), "=f"(b) : "r"(hi), "f"(x), "f"(y));
  lo = pack_f16(a, b);
}
// the same after multiplication with f = (f, f)
__device__ __forceinline__ void split2_scaled(uint32_t x, uint32_t y, uint64_t f, uint32_t& hi, uint32_t& lo) {
  float a, b;
  unpair(mul2(pair_of(__uint_as_float(x), __uint_as_float(y)), f), a, b);
  split2(a, b, hi, lo);
}
// packed limbs -> the two values
__device__ __forceinline__ float2 join2(uint32_t hi, uint32_t lo) {
  const float2 h = unpack_f16(hi);
  float2 v;
  asm("{\n\t.reg .b16 l0, l1;\n\tmov.b32 {l0, l1}, %2;\n\tadd.rn.f32.f16 %0, l0, %3;\n\tadd.rn.f32.f16 %1, l1, %4;\n\t}"
      : "=f"(v.x), "=f"(v.y) : "r"(lo), "f"(h.x), "f"(h.y));
  return v;
}
// row r, 16-byte chunk c of a panel
__device__ __forceinline__ uint32_t at_chunk(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

}  // namespace
