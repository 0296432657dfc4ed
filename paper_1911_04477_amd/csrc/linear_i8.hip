// int8 matrix product with a scale per row of either operand (bnn_linear_i8).
#include "few_mm.h"
#include "float_types.h"

namespace bnn {

// y = (float)sum * sa[m] * sb[n] + bias[n]: the 32-bit sum is exact, fp32 from there, one rounding to the output's type.
struct LinearEpilogue {
  const float *sa, *sb, *bias;
  void *y;
  int64_t ldy;
  int type;
  using Row = float;
  struct Columns {
    f32x4 scale, bias;
  };
  __device__ __forceinline__ Row row(int m) const { return sa[m]; }
  __device__ __forceinline__ Columns columns(int n, int N) const {
    return {load4(sb, n, N), bias ? load4(bias, n, N) : f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
  }
  __device__ __forceinline__ void operator()(int m, int n, int N, Row a, const Columns &c, const v4i &sum) const {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmaf((float)sum[i] * a, c.scale[i], c.bias[i]);
    if (type == BNN_BF16) store4(static_cast<__bf16 *>(y) + m * ldy, n, N, v);
    else if (type == BNN_F16) store4(static_cast<_Float16 *>(y) + m * ldy, n, N, v);
    else store4(static_cast<float *>(y) + m * ldy, n, N, v);
  }
  template <class F>
  bnn_status fixed(const F &f) const { return f(*this); }
};

}  // namespace bnn

extern "C" bnn_status bnn_linear_i8(const int8_t *a, int64_t lda, const float *a_scale, const int8_t *b, int64_t ldb,
                                    const float *b_scale, const float *bias, int64_t M, int64_t N, int64_t K, void *y,
                                    int type, int64_t ldy, void *stream) {
  using namespace bnn;
  if (M < 0 || N < 0 || K <= 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (lda < K || ldb < K || ldy < N) return BNN_ERR_STRIDE;
  if (K > 131071 || M > INT32_MAX - 256 || N > INT32_MAX - 256) return BNN_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return BNN_OK;
  if (!a || !a_scale || !b || !b_scale || !y) return BNN_ERR_NULL;
  if (!aligned16(a) || !aligned16(a_scale) || !aligned16(b) || !aligned16(b_scale) || !aligned16(bias) || !aligned16(y))
    return BNN_ERR_ALIGN;
  MmOperands p = {};
  p.A = reinterpret_cast<const char *>(a);
  p.B0 = p.B1 = reinterpret_cast<const char *>(b);
  p.lda = lda, p.ldb0 = p.ldb1 = ldb;
  p.M = (int)M, p.N = (int)N, p.kbytes = (int)K;
  p.dma = mm_dma(a, lda) && mm_dma(b, ldb);
  const LinearEpilogue epi = {a_scale, b_scale, bias, y, ldy, type};
  return run_product<MM_I8, false>(p, epi, KID_LINEAR_I8_FEW, KID_LINEAR_I8, static_cast<hipStream_t>(stream));
}
