// Device helpers of the dense operators: 16- and 32-bit element types, the
// activations with their slopes.
#pragma once
#include "common.hpp"
#include "dense.hpp"

namespace moe {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <class E> struct Vec8;
template <> struct Vec8<bf16_t> { typedef bf16x8 type; };
template <> struct Vec8<f16_t> { typedef f16x8 type; };

// Eight consecutive elements (16-byte aligned) to fp32 and back, rounded to
// nearest even.
template <class E>
__device__ __forceinline__ f32x8 load8(const E* p) {
  if constexpr (__is_same(E, float)) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else {
    return __builtin_convertvector(*reinterpret_cast<const typename Vec8<E>::type*>(p), f32x8);
  }
}
template <class E>
__device__ __forceinline__ void store8(E* p, const f32x8& v) {
  if constexpr (__is_same(E, float)) {
    *reinterpret_cast<f32x4*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    *reinterpret_cast<f32x4*>(p + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
  } else {
    *reinterpret_cast<typename Vec8<E>::type*>(p) = __builtin_convertvector(v, typename Vec8<E>::type);
  }
}

// D(32x32, fp32) += A(32x16) * B(16x32); fragments and D as mfma32x32x16.
template <class E>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c) {
  if constexpr (__is_same(E, bf16_t)) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// D(16x16, fp32) += A(16x32) * B(32x16); fragments and D as mfma16x16x32.
template <class E>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c) {
  if constexpr (__is_same(E, bf16_t)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 1 / (1 + exp(-z)) with the hardware reciprocal (about 1 ulp); exp overflowing
// gives 0, as it should.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// SiLU: a = g s, slope s (1 + g (1 - s)) with s = logistic(g).
// GELU (tanh form): 0.5 (1 + tanh z) = logistic(2 z), z = c (g + 0.044715 g^3),
// c = sqrt(2 / pi): a = g s, slope s + g s (1 - s) 2 c (1 + 3 * 0.044715 g^2).
// Past |g| = 16 that logistic is 0 or 1 in fp32, so its argument and g times the
// argument's slope (gdz) are taken there.  A NaN stays one, in the slope too.
constexpr float kGelu2C = 1.5957691216057308f, kGeluA = 0.044715f;
__device__ __forceinline__ float act_arg(int act, float g, float& gdz) {
  if (act == kSilu) {
    gdz = g;
    return g;
  }
  const float c = g > 16.0f ? 16.0f : g < -16.0f ? -16.0f : g, q = kGeluA * c * c, k = kGelu2C * c;
  gdz = k * fmaf(3.0f, q, 1.0f);
  return k * (q + 1.0f);
}
__device__ __forceinline__ float act_of(int act, float g) {
  float gdz;
  return g * logistic(act_arg(act, g, gdz));
}
__device__ __forceinline__ void act_and_slope(int act, float g, float& a, float& slope) {
  float gdz;
  const float s = logistic(act_arg(act, g, gdz));
  a = g * s;
  slope = s * fmaf(gdz, 1.0f - s, 1.0f);
}

}  // namespace moe
