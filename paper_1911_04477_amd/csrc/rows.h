// Rows of a matrix over the threads of a team: eight consecutive values a thread and piece, read and written at any
// alignment, sums and maxima over a row, and a row's 8-bit form.
#pragma once
#include "float_types.h"

namespace bnn {

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

// Where a thread's eight values of a row of D lie: values c .. c + 7, read from `at` on, inside the row, and then moved down
// by `shift` (8 and more: none is left).  Loads under a condition of their own would each wait for the one before; so all of
// a row's loads are issued first, without one, and only threads at the end of a row move what they got.
enum RowEdge : int {
  EDGE_WHOLE = 0,   // D a multiple of eight: a thread has all of its values or none
  EDGE_RAGGED = 1,  // D > 8
  EDGE_SMALL = 2    // D < 8, read one by one
};
inline RowEdge row_edge(int64_t D) { return D % 8 == 0 ? EDGE_WHOLE : D > 8 ? EDGE_RAGGED : EDGE_SMALL; }
template <int EDGE>
struct Place8 {
  int c, at, shift;
  __device__ __forceinline__ Place8(int c_, int D) : c(c_), at(EDGE == EDGE_SMALL ? 0 : min(c_, D - 8)), shift(c_ - at) {}
};
template <class E>
struct Piece8 {
  typedef E E8 __attribute__((ext_vector_type(8)));
  E8 v;
  template <int EDGE>
  __device__ __forceinline__ void load(const E *row, const Place8<EDGE> &p, int D) {
    if constexpr (EDGE == EDGE_SMALL) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = row[min(i, D - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= D) v[i] = (E)0.0f;
    } else if constexpr (sizeof(E) == 4) {
      typedef E E4 __attribute__((ext_vector_type(4)));
      const auto lo = __builtin_bit_cast(E4, *reinterpret_cast<const u32x4_any *>(row + p.at));
      const auto hi = __builtin_bit_cast(E4, *reinterpret_cast<const u32x4_any *>(row + p.at + 4));
      v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      v = __builtin_bit_cast(E8, *reinterpret_cast<const u32x4_any *>(row + p.at));
    }
  }
  // After the loads: the values that belong here, zeros behind them.
  template <int EDGE>
  __device__ __forceinline__ void settle(const Place8<EDGE> &p) {
    const E8 none = {};
    const int shift = EDGE == EDGE_RAGGED ? p.shift : 0;
    if (shift & 4) v = __builtin_shufflevector(v, none, 4, 5, 6, 7, 8, 9, 10, 11);
    if (shift & 2) v = __builtin_shufflevector(v, none, 2, 3, 4, 5, 6, 7, 8, 9);
    if (shift & 1) v = __builtin_shufflevector(v, none, 1, 2, 3, 4, 5, 6, 7, 8);
    if (p.shift >= 8) v = none;
  }
  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (E)x;
  }
};
// The same where nothing else is to be requested at once.
template <class E>
__device__ __forceinline__ void load8(float (&v)[8], const E *row, int c, int D) {
  Piece8<E> x;
  if (D >= 8) {
    const Place8<EDGE_RAGGED> p(c, D);
    x.load(row, p, D);
    if (p.shift) x.settle(p);
  } else {
    const Place8<EDGE_SMALL> p(c, D);
    x.load(row, p, D);
    if (p.shift) x.settle(p);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)x.v[i];
}

template <class E>
__device__ __forceinline__ void store8(E *row, int c, int D, const float (&v)[8]) {
  typedef E E8 __attribute__((ext_vector_type(8)));
  typedef E E4 __attribute__((ext_vector_type(4)));
  if (c + 8 <= D) {
    if constexpr (sizeof(E) == 4) {
      *reinterpret_cast<u32x4_any *>(row + c) = __builtin_bit_cast(u32x4, (E4{(E)v[0], (E)v[1], (E)v[2], (E)v[3]}));
      *reinterpret_cast<u32x4_any *>(row + c + 4) = __builtin_bit_cast(u32x4, (E4{(E)v[4], (E)v[5], (E)v[6], (E)v[7]}));
    } else {
      E8 x;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (E)v[i];
      *reinterpret_cast<u32x4_any *>(row + c) = __builtin_bit_cast(u32x4, x);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < D) row[c + i] = (E)v[i];
  }
}

// Sums and maxima over a team: one wave, or (BLOCK) all waves of a workgroup, the same order at every call.  Within a wave
// by lane exchanges of the vector unit: rows of 16 lanes, then the rows, the result from the last lane.  0 is neutral.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t other_lane(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
template <class Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, const Op &op) {
  x = op(x, other_lane<0x111, 0xf>(x));
  x = op(x, other_lane<0x112, 0xf>(x));
  x = op(x, other_lane<0x114, 0xf>(x));
  x = op(x, other_lane<0x118, 0xf>(x));
  x = op(x, other_lane<0x142, 0xa>(x));
  x = op(x, other_lane<0x143, 0xc>(x));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// V values at once.  lds: V * 16 words that no other reduction uses that threads could still be reading; words of waves
// that the workgroup does not have are 0 (clear_words).
template <bool BLOCK, int V, class Op>
__device__ __forceinline__ void team_reduce(uint32_t (&x)[V], uint32_t *lds, const Op &op) {
#pragma unroll
  for (int k = 0; k < V; ++k) x[k] = wave_reduce(x[k], op);
  if constexpr (BLOCK) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < V; ++k) lds[k * 16 + (threadIdx.x >> 6)] = x[k];
    __syncthreads();
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int k = 0; k < V; ++k) {
      x[k] = 0u;
      for (int w = 0; w < (int)(blockDim.x >> 6); w += 4) {
        const Words v = *reinterpret_cast<const Words *>(lds + k * 16 + w);
        x[k] = op(x[k], op(op(v[0], v[1]), op(v[2], v[3])));
      }
    }
  }
}
template <bool BLOCK, int V>
__device__ __forceinline__ void team_sum(float (&x)[V], uint32_t *lds) {
  uint32_t u[V];
#pragma unroll
  for (int k = 0; k < V; ++k) u[k] = __float_as_uint(x[k]);
  team_reduce<BLOCK>(u, lds, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); });
#pragma unroll
  for (int k = 0; k < V; ++k) x[k] = __uint_as_float(u[k]);
}
template <bool BLOCK>
__device__ __forceinline__ float team_sum(float x, uint32_t *lds) {
  float v[1] = {x};
  team_sum<BLOCK>(v, lds);
  return v[0];
}
// Of magnitudes, as bit patterns: a NaN is larger than infinity, and stays.
template <bool BLOCK>
__device__ __forceinline__ float team_max_magnitude(uint32_t bits, uint32_t *lds) {
  uint32_t v[1] = {bits};
  team_reduce<BLOCK>(v, lds, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  return __uint_as_float(v[0]);
}
template <int N>
__device__ __forceinline__ void clear_words(uint32_t (&lds)[N]) {
  for (int i = threadIdx.x; i < N; i += blockDim.x) lds[i] = 0u;
  __syncthreads();
}

// Threads a row of D values, NV pieces of eight each: whole waves.
inline int row_threads(int64_t D, int NV) { return (int)((D + 8ll * NV * 64 - 1) / (8ll * NV * 64)) * 64; }

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
