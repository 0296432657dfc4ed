// Floating-point element types of the quantised and gated layers: conversion to fp32 and, rounded to nearest even, back.
#pragma once
#include "common.h"

namespace bnn {

inline bool float_type(int t) { return t == BNN_F32 || t == BNN_BF16 || t == BNN_F16; }
inline int float_size(int t) { return t == BNN_F32 ? 4 : 2; }

// n workgroups of at most 1024 threads.  A launch counts the threads of a dimension in 32 bits, and drops what is above them without an
// error; so from 2^20 workgroups on they lie in two dimensions, and some of the last row have nothing to do (wide_grid).  Kernels
// that would wait for their arguments to know that are launched again instead (wide_launches).
constexpr int64_t WIDE_ROW = 1 << 20;
inline dim3 wide_grid(int64_t n) {
  return n <= WIDE_ROW ? dim3((uint32_t)n) : dim3((uint32_t)WIDE_ROW, (uint32_t)((n - 1) / WIDE_ROW + 1));
}
__device__ __forceinline__ int64_t wide_block() { return blockIdx.y * WIDE_ROW + blockIdx.x; }
template <class F>
void wide_launches(int64_t n, const F &launch) {  // launch(first, workgroups)
  for (int64_t first = 0; first < n; first += WIDE_ROW) launch(first, (uint32_t)(n - first < WIDE_ROW ? n - first : WIDE_ROW));
}

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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));  // global loads and stores take any byte address

// 16 bytes of a row of `end` bytes from byte k on, zeros past its end, any alignment; nothing is read outside the row.  Of a
// row's last piece the 16 bytes that end with the row, moved (element by element only in rows of less than 16 bytes: loads
// under a mask each wait for the one before).
template <class E>
__device__ __forceinline__ u32x4 bytes16(const char *row, int k, int end) {
  if (k + 16 <= end) return *reinterpret_cast<const u32x4_any *>(row + k);
  u32x4 v = {0u, 0u, 0u, 0u};
  if (k >= end) return v;
  if (end >= 16) {
    const u32x4 last = *reinterpret_cast<const u32x4_any *>(row + end - 16);
    uint64_t lo = last[0] | (uint64_t)last[1] << 32, hi = last[2] | (uint64_t)last[3] << 32;
    const int bits = 8 * (k + 16 - end);  // 8 .. 120
    lo = bits < 64 ? lo >> bits | hi << (64 - bits) : hi >> (bits - 64);
    hi = bits < 64 ? hi >> bits : 0u;
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
#pragma unroll
  for (int e = 0; e < 16 / (int)sizeof(E); ++e) {
    if (k + e * (int)sizeof(E) < end) {
      uint32_t x;
      if constexpr (sizeof(E) == 1) x = *reinterpret_cast<const uint8_t *>(row + k + e);
      else if constexpr (sizeof(E) == 2) x = *reinterpret_cast<const uint16_t *>(row + k + 2 * e);
      else x = *reinterpret_cast<const uint32_t *>(row + k + 4 * e);
      v[e * sizeof(E) / 4] |= x << (8 * (e * sizeof(E) % 4));
    }
  }
  return v;
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
