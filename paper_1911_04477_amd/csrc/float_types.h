// Floating-point element types of the quantised and gated layers: conversion to fp32 and, rounded to nearest even, back.
#pragma once
#include "common.h"

namespace bnn {

inline bool float_type(int t) { return t == BNN_F32 || t == BNN_BF16 || t == BNN_F16; }
inline int float_size(int t) { return t == BNN_F32 ? 4 : 2; }

template <int DT>
struct Float;
template <>
struct Float<BNN_F32> { using type = float; };
template <>
struct Float<BNN_BF16> { using type = __bf16; };
template <>
struct Float<BNN_F16> { using type = _Float16; };

// Calls f with the element type as a tag, f(Float<..>()).
template <class F>
inline auto with_float(int t, const F &f) {
  if (t == BNN_F32) return f(Float<BNN_F32>());
  if (t == BNN_BF16) return f(Float<BNN_BF16>());
  return f(Float<BNN_F16>());
}

// Values n .. n + 3 of an aligned vector of N, zeros past its end; n is a multiple of 4.
typedef float f32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4 load4(const float *v, int n, int N) {
  if (n + 4 <= N) return *reinterpret_cast<const f32x4 *>(v + n);
  return f32x4{v[n], n + 1 < N ? v[n + 1] : 0.0f, n + 2 < N ? v[n + 2] : 0.0f, 0.0f};
}
struct NoConstants {};

// Four consecutive values of a row of N, from column n on; whole groups go out as one store, which takes any alignment.
template <class E, class V>
__device__ __forceinline__ void store4(E *row, int n, int N, const V &v) {
  typedef E E4 __attribute__((ext_vector_type(4)));
  typedef uint32_t Words __attribute__((ext_vector_type(sizeof(E)), aligned(1)));
  if (n + 4 <= N) {
    E4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (E)v[i];
    *reinterpret_cast<Words *>(row + n) = __builtin_bit_cast(Words, o);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) row[n + i] = (E)v[i];
  }
}

}  // namespace bnn
