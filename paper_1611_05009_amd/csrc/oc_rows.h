// Element types of row operators: eight elements per lane, read and written
// as one vector where the rows allow it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ocr {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x8 = __attribute__((ext_vector_type(8), aligned(16))) float;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;

// Eight bits: 4 of exponent, 3 of mantissa, no infinity, up to 448.
struct e4m3 {
  uint8_t bits;
};

template <class T>
struct Vec8;
template <>
struct Vec8<float> {
  using type = f32x8;
};
template <>
struct Vec8<__bf16> {
  using type = bf16x8;
};
template <>
struct Vec8<_Float16> {
  using type = f16x8;
};

__device__ __forceinline__ f32x8 load8(const float* p) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <class T>
__device__ __forceinline__ f32x8 load8(const T* p) {
  return __builtin_convertvector(*(const typename Vec8<T>::type*)p, f32x8);
}

__device__ __forceinline__ void store8(float* p, f32x8 x) {
  *(f32x4*)p = __builtin_shufflevector(x, x, 0, 1, 2, 3);
  *(f32x4*)(p + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
}
// The packed conversion rounds to nearest even.
__device__ __forceinline__ void store8(e4m3* p, f32x8 x) {
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], a, true);
  int b = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], b, true);
  *(u32x2*)p = u32x2{(uint32_t)a, (uint32_t)b};
}
template <class T>
__device__ __forceinline__ void store8(T* p, f32x8 x) {
  *(typename Vec8<T>::type*)p = __builtin_convertvector(x, typename Vec8<T>::type);
}

template <class T>
__device__ __forceinline__ void store1(T* p, float x) {
  *p = (T)x;
}
__device__ __forceinline__ void store1(e4m3* p, float x) {
  p->bits = (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 255);
}

// Sum or maximum over aligned groups of `width` lanes (a power of two, at
// most 64).
__device__ __forceinline__ float group_sum(float x, int width) {
  for (int i = width >> 1; i; i >>= 1) x += __shfl_xor(x, i);
  return x;
}
__device__ __forceinline__ float group_max(float x, int width) {
  for (int i = width >> 1; i; i >>= 1) x = fmaxf(x, __shfl_xor(x, i));
  return x;
}

}  // namespace ocr
