// Element types of feature rows, as the row-wise kernels read and write them.
#pragma once

#include "common.h"

namespace spc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two float32 values as one word of a 16-bit type, each rounded to nearest even.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<_Float16>(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}
template <>
__device__ __forceinline__ uint32_t pack2<__bf16>(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
template <typename T>
__device__ __forceinline__ void unpack2(uint32_t w, float* a, float* b);
template <>
__device__ __forceinline__ void unpack2<_Float16>(uint32_t w, float* a, float* b) {
  const f16x2 v = __builtin_bit_cast(f16x2, w);
  *a = (float)v[0];
  *b = (float)v[1];
}
template <>
__device__ __forceinline__ void unpack2<__bf16>(uint32_t w, float* a, float* b) {
  *a = __builtin_bit_cast(float, w << 16);
  *b = __builtin_bit_cast(float, w & 0xFFFF0000u);
}

// Eight consecutive elements of a row: one 16-byte access in 16-bit types, two in float32.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(a[i], &v[2 * i], &v[2 * i + 1]);
  }
}
// Stored past the caches: rows that no other workgroup reads.
template <typename T>
__device__ __forceinline__ void store8_past(T* p, const float* v) {
  if constexpr (sizeof(T) == 4) {
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4*>(p) + 1);
  } else {
    const u32x4 w = {pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
  }
}

// Four float32 values as e4m3 (OCP: 3 mantissa bits, largest 448), rounded to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// Blocks of an 8-bit row that share one scale, and the scale of a block whose largest
// magnitude is `top`: at least 2^-126, so that a block of zeros has a finite inverse.
constexpr int kScaleBlock = 128;
__device__ __forceinline__ float block_scale(float top) { return fmaxf(top / 448.0f, 0x1p-126f); }

}  // namespace spc
