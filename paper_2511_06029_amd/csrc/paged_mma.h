// Storage types of the paged cache on the matrix cores: operand vectors,
// products and transposing LDS reads of bf16 and fp16.
#pragma once

#include "device_common.h"

namespace lethe {

typedef float mma_f32x4_t __attribute__((ext_vector_type(4)));
typedef float mma_f32x16_t __attribute__((ext_vector_type(16)));
typedef float mma_f32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_cvoid;

// Whether a 16-bit half of v has all bits of the exponent e.
__device__ inline bool mma_odd(const uint4& v, uint32_t e) {
  auto odd = [&](uint32_t u) { return (u & e) == e || ((u >> 16) & e) == e; };
  return odd(v.x) || odd(v.y) || odd(v.z) || odd(v.w);
}

template <typename T>
struct Mma;

template <>
struct Mma<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  // Whether one of eight elements is an infinity or NaN.
  static __device__ inline bool odd(const uint4& v) { return mma_odd(v, 0x7f80u); }
  static __device__ inline mma_f32x4_t mma16(x8 a, x8 b, mma_f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ inline mma_f32x16_t mma32(x8 a, x8 b, mma_f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ inline x4 read_tr(const lds_char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) x4*)p);
  }
};

template <>
struct Mma<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x4 __attribute__((ext_vector_type(4)));
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static __device__ inline bool odd(const uint4& v) { return mma_odd(v, 0x7c00u); }
  static __device__ inline mma_f32x4_t mma16(x8 a, x8 b, mma_f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ inline mma_f32x16_t mma32(x8 a, x8 b, mma_f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ inline x4 read_tr(const lds_char* p) {
    typedef __fp16 h4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) h4*)p));
  }
};

template <typename T>
__device__ inline typename Mma<T>::x8 mma_zero() {
  return __builtin_bit_cast(typename Mma<T>::x8, make_uint4(0, 0, 0, 0));
}

}  // namespace lethe
