// Rows of a matrix over the threads of a team: eight consecutive values a thread and piece, read and written at any
// alignment, sums and maxima over a row, and a row's 8-bit form.
#pragma once
#include "float_types.h"

namespace bnn {

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x4_row __attribute__((ext_vector_type(4), aligned(1)));

// Values c .. c + 7 of a row of D, zeros past its end.
template <class E>
__device__ __forceinline__ void load8(float (&v)[8], const E *row, int c, int D) {
  typedef E E8 __attribute__((ext_vector_type(8)));
  typedef E E4 __attribute__((ext_vector_type(4)));
  if (c + 8 <= D) {
    if constexpr (sizeof(E) == 4) {
      const auto lo = __builtin_bit_cast(E4, *reinterpret_cast<const u32x4_row *>(row + c));
      const auto hi = __builtin_bit_cast(E4, *reinterpret_cast<const u32x4_row *>(row + c + 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (float)lo[i], v[4 + i] = (float)hi[i];
    } else {
      const auto x = __builtin_bit_cast(E8, *reinterpret_cast<const u32x4_row *>(row + c));
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < D ? (float)row[c + i] : 0.0f;
  }
}

template <class E>
__device__ __forceinline__ void store8(E *row, int c, int D, const float (&v)[8]) {
  typedef E E8 __attribute__((ext_vector_type(8)));
  typedef E E4 __attribute__((ext_vector_type(4)));
  if (c + 8 <= D) {
    if constexpr (sizeof(E) == 4) {
      *reinterpret_cast<u32x4_row *>(row + c) = __builtin_bit_cast(u32x4_row, (E4{(E)v[0], (E)v[1], (E)v[2], (E)v[3]}));
      *reinterpret_cast<u32x4_row *>(row + c + 4) = __builtin_bit_cast(u32x4_row, (E4{(E)v[4], (E)v[5], (E)v[6], (E)v[7]}));
    } else {
      E8 x;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (E)v[i];
      *reinterpret_cast<u32x4_row *>(row + c) = __builtin_bit_cast(u32x4_row, x);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < D) row[c + i] = (E)v[i];
  }
}

// Sum or maximum over a team of T threads (a wave, or a whole workgroup), the same order at every call.  `lds` holds
// T / 64 values and is not used by another reduction that threads could still be reading.
template <int T, class Op>
__device__ __forceinline__ uint32_t team_reduce(uint32_t x, uint32_t *lds, const Op &op) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = op(x, (uint32_t)__shfl_xor((int)x, d));
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) x = op(x, lds[w]);
  }
  return x;
}
template <int T>
__device__ __forceinline__ float team_sum(float x, uint32_t *lds) {
  return __uint_as_float(team_reduce<T>(__float_as_uint(x), lds, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
// Of magnitudes, as bit patterns: a NaN is larger than infinity, and stays.
template <int T>
__device__ __forceinline__ float team_max_magnitude(uint32_t bits, uint32_t *lds) {
  return __uint_as_float(team_reduce<T>(bits, lds, [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A row's 8-bit form: s = a / 127 and q = rint(x * (127 / a)) with a the row's largest magnitude, both quotients
// correctly rounded, so that q and s do not depend on how the row was read.  Rows below 2^-100 count as zero (127 / a
// could overflow).  A row that holds an infinity or a NaN has q = 0 and its largest magnitude as scale, NaN before
// infinity: what is multiplied with it becomes NaN instead of a number that hides it.
struct RowScale {
  float scale, inv;
};
__device__ __forceinline__ RowScale row_scale(float a) {
  if (!(a < __builtin_inff())) return {a, 0.0f};
  if (a < 0x1p-100f) return {0.0f, 0.0f};
  return {a / 127.0f, 127.0f / a};
}
__device__ __forceinline__ void store_q8(int8_t *row, int c, int D, const float (&v)[8], float inv) {
  uint32_t q[2] = {0u, 0u};
  if (inv != 0.0f) {  // |x * inv| <= 127 but for the rounding of the product, which rint takes back
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i / 4] |= ((uint32_t)(int)rintf(v[i] * inv) & 0xffu) << (8 * (i % 4));
  }
  if (c + 8 <= D) {
    *reinterpret_cast<u32x2_any *>(row + c) = u32x2_any{q[0], q[1]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < D) row[c + i] = (int8_t)(q[i / 4] >> (8 * (i % 4)));
  }
}

}  // namespace bnn
