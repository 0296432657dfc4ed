// 8-bit floating point with block scales: e4m3 values (four bits of exponent, three of mantissa, the largest 448) in blocks of
// 128 along a row, each with a power of two as scale, kept as the byte p + 127.  The matrix instruction takes such bytes with its
// operands, so a product needs no multiplications of its own for them; and a power of two changes no digit of a value, so
// that the quantised values are the values rounded once.
#pragma once
#include "rows.h"

namespace bnn {

constexpr int F8_BLOCK = 128;
inline int64_t f8_row_bytes(int64_t K) { return (K + F8_BLOCK - 1) / F8_BLOCK * F8_BLOCK; }
inline int64_t f8_blocks(int64_t K) { return (K + F8_BLOCK - 1) / F8_BLOCK; }
inline int64_t f8_scale_bytes(int64_t K) { return (f8_blocks(K) + 3) / 4 * 4; }

// The least p >= -100 with a <= 448 * 2^p, as p + 127; a is the bit pattern of a finite magnitude.  448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t a) {
  const int p = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(p, 27);
}
// 2^-p from p + 127 = 27 .. 247
__device__ __forceinline__ float f8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// A magnitude's bits, or 0 for an infinity or a NaN: these do not count for a block's scale.
__device__ __forceinline__ uint32_t f8_magnitude(float x) {
  const uint32_t m = magnitude(x);
  return m < 0x7f800000u ? m : 0u;
}
// Four values, already times 2^-p, as bytes: rounded to nearest, ties to even; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t f8_pack(float a, float b, float c, float d) {
  const float none = __builtin_nanf("");
  a = fabsf(a) <= 448.0f ? a : none, b = fabsf(b) <= 448.0f ? b : none;
  c = fabsf(c) <= 448.0f ? c : none, d = fabsf(d) <= 448.0f ? d : none;
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// The largest of a row of 16 lanes, in all of them.
__device__ __forceinline__ uint32_t row16_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));  // turned by 8, 4, 2, 1 lanes
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));
  return x;
}

// Sixteen lanes' eight values each, a whole block, to a row of e4m3 and its scale; `c`: of a lane's first value.  Values past the
// row's end are zeros by now.
__device__ __forceinline__ void f8_store_block(const float (&v)[8], uint8_t *q, uint8_t *scale, int c) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, f8_magnitude(v[i]));
  const uint32_t byte = f8_scale_byte(row16_max(top));
  const float inv = f8_inverse(byte);
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  *reinterpret_cast<u32x2 *>(q + c) = u32x2{f8_pack(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                                            f8_pack(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
  if ((c & 127) == 0) scale[c >> 7] = (uint8_t)byte;
}

// The longest row that products take: whole blocks at a stride below 2^22.
constexpr int64_t F8_MOST_K = (1 << 22) - F8_BLOCK;

// What operands in this form have to be: rows of whole blocks on 16 bytes, offsets inside a tile of 256 rows in 32 bits.
inline bnn_status f8_check(const void *q, int64_t ld, const void *scale, int64_t scale_ld, int64_t K, bool products = true) {
  if (ld < f8_row_bytes(K) || scale_ld < f8_scale_bytes(K)) return BNN_ERR_STRIDE;
  if (ld % 16 || scale_ld % 4) return BNN_ERR_STRIDE;
  if (products && (ld >= (1 << 22) || scale_ld >= (1 << 22))) return BNN_ERR_UNSUPPORTED;
  if (!q || !scale) return BNN_ERR_NULL;
  if (!aligned16(q) || !aligned4(scale)) return BNN_ERR_ALIGN;
  return BNN_OK;
}

}  // namespace bnn
