// The 8-bit block-scaled cache format (JF_FMT_E4M3_B32): e4m3 codes and one
// power-of-two scale 2^e per block of 32 positions and KV head, for K and V
// apart.  Shared by the append, read, decode, prefill and eviction kernels.
#pragma once
#include "common.cuh"

namespace jfkv {

constexpr int KV8_BLOCK = 32;    // positions that share a scale
constexpr int KV8_EMIN = -40;    // range of the exponents: a call's scores, weights and
constexpr int KV8_EMAX = 40;     // sums then stay inside fp32 whatever blocks meet in it

__host__ __device__ __forceinline__ int clamp_exp8(int e) {
  return e < KV8_EMIN ? KV8_EMIN : (e > KV8_EMAX ? KV8_EMAX : e);
}

// Smallest e with amax <= 448 * 2^e (448 = 1.75 * 2^8 is the largest e4m3
// value), limited to the range above; amax finite and >= 0.
__device__ __forceinline__ int exp8_of(float amax) {
  const uint32_t b = __float_as_uint(amax);
  return clamp_exp8((int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// Exponent of a stored scale word; any bits (a slot nothing wrote) give one
// inside the range.
__device__ __forceinline__ int exp8_of_scale(float s) {
  return clamp_exp8((int)((__float_as_uint(s) >> 23) & 0xFFu) - 127);
}

// 2^e for e inside a normal fp32's range
__device__ __forceinline__ float two8(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// two values -> two e4m3 codes (round to nearest even, saturating; NaN stays
// NaN), lo in the low byte
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// the codes of the low (high) half of a word -> f16x2, exact
__device__ __forceinline__ void f16x4_of_e4m3(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\n"
      "cvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
      : "=r"(lo), "=r"(hi) : "r"(w));
}

__device__ __forceinline__ float2 f32x2_of_f16x2(uint32_t h) {
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

__device__ __forceinline__ uint32_t pack_bf16x2_rn(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Codes rounded again for a scale 2^-s times as large (value = code * 2^s under
// the new scale, at most 448).  In fp16: products of at least 2^-10, half the
// smallest code, are exact, and smaller ones become zero either way; s < -24
// leaves only those.
__device__ __forceinline__ uint32_t f16x2_two(int s) {
  const __half2 h = __float2half2_rn(s < -24 ? 0.f : two8(s));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t e4m3x4_of_f16x2(uint32_t lo, uint32_t hi) {
  uint32_t r;
  asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n"
      "cvt.rn.satfinite.e4m3x2.f16x2 b, %2;\nmov.b32 %0, {a, b};\n}\n"
      : "=r"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int N>
__device__ __forceinline__ void rescale_f16(uint32_t (&v)[N], int s) {
  if (s > 15) {   // past fp16's powers of two
    const uint32_t p = f16x2_two(15);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = mul_f16x2(v[i], p);
    // what is left: a code above zero is at least 2^-9 and its value at most 448, so s <= 17;
    // zeros come with any s, and have to meet a finite power to stay zeros
    s = min(s - 15, 15);
  }
  const uint32_t p = f16x2_two(s);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = mul_f16x2(v[i], p);
}
__device__ __forceinline__ uint32_t rescale_e4m3x4(uint32_t w, int s) {
  uint32_t v[2];
  f16x4_of_e4m3(w, v[0], v[1]);
  rescale_f16(v, s);
  return e4m3x4_of_f16x2(v[0], v[1]);
}

}  // namespace jfkv
