// Gated feed-forward, h = act(x Wg^T) * (x Wu^T): both projections, the activation and the product in one kernel, from
// 16-bit floating-point operands (with its backward pass) or from 8-bit ones with scales.
#include <algorithm>

#include "few_mm.h"
#include "float_types.h"

namespace bnn {

// The activation, or with SLOPE also its derivative.  exp and the quotient are the hardware's (relative error of a few
// 2^-24; what exp loses for large arguments belongs to values next to zero).
template <bool SLOPE>
__device__ __forceinline__ float activation(int act, float z, float &slope) {
  constexpr float LOG2E = 1.44269504088896341f;
  float a;
  if (act == BNN_ACT_SILU) {
    const float t = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -LOG2E));
    a = z * t;
    if (SLOPE) slope = t * (1.0f + z * (1.0f - t));
  } else if (act == BNN_ACT_GELU) {
    const float t = 0.5f * erfcf(z * -0.70710678118654752f);  // of the normal distribution, without cancellation below 0
    a = z * t;
    if (SLOPE) slope = t + z * 0.39894228040143268f * __builtin_amdgcn_exp2f(z * z * (-0.5f * LOG2E));
  } else if (act == BNN_ACT_GELU_TANH) {
    const float k = 0.79788456080286536f, c = 0.044715f;
    const float t = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-2.0f * LOG2E * k * (z + c * z * z * z)));  // (1 + tanh) / 2
    a = z * t;
    if (SLOPE) slope = t + 2.0f * z * t * (1.0f - t) * k * (1.0f + 3.0f * c * fminf(z * z, 1e30f));
  } else {
    a = z > 0.0f || z != z ? z : 0.0f;
    if (SLOPE) slope = z > 0.0f ? 1.0f : 0.0f;
  }
  return a;
}

// Where a backward pass will follow, `saved` takes what it multiplies the gradient of h with, in fp32 (16 bits would round
// the gradients of the projections twice): act'(g) * u for that of g = x Wg^T, act(g) for that of u = x Wu^T.
template <class E>
struct GatedEpilogue {
  E *h;
  int64_t ldh;
  float *saved;
  int64_t plane;  // values in one of the two
  int act, vec, savedVec;
  using Row = NoConstants;
  __device__ __forceinline__ Row row(int) const { return {}; }
  __device__ __forceinline__ NoConstants columns(int, int) const { return {}; }
  __device__ __forceinline__ void operator()(int m, int n, int N, Row, NoConstants, const v4f &g, const v4f &u) const {
    float o[4], dg[4], du[4];
    if (saved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float slope;
        du[i] = activation<true>(act, g[i], slope);
        dg[i] = slope * u[i];
        o[i] = du[i] * u[i];
      }
      store4(saved + (int64_t)m * N, n, N, dg, savedVec);
      store4(saved + plane + (int64_t)m * N, n, N, du, savedVec);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float none;
        o[i] = activation<false>(act, g[i], none) * u[i];
      }
    }
    store4(h + m * ldh, n, N, o, vec);
  }
};

struct GatedI8Epilogue {
  const float *sx, *sg, *su;
  void *h;
  int64_t ldh;
  int type, act, vec;
  using Row = float;
  struct Columns {
    f32x4 g, u;
  };
  __device__ __forceinline__ Row row(int m) const { return sx[m]; }
  __device__ __forceinline__ Columns columns(int n, int N) const { return {load4(sg, n, N), load4(su, n, N)}; }
  __device__ __forceinline__ void operator()(int m, int n, int N, Row a, const Columns &c, const v4i &g, const v4i &u) const {
    float o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float none;
      o[i] = activation<false>(act, (float)g[i] * a * c.g[i], none) * ((float)u[i] * a * c.u[i]);
    }
    if (type == BNN_BF16) store4(static_cast<__bf16 *>(h) + m * ldh, n, N, o, vec);
    else if (type == BNN_F16) store4(static_cast<_Float16 *>(h) + m * ldh, n, N, o, vec);
    else store4(static_cast<float *>(h) + m * ldh, n, N, o, vec);
  }
};

// A plain product, rounded to the operands' type; rows from `split` on go to a second matrix.
template <class E>
struct ProductEpilogue {
  E *y0, *y1;
  int64_t ld0, ld1;
  int rows0, split, vec;  // rows0 <= split: rows between them are padding
  using Row = NoConstants;
  __device__ __forceinline__ Row row(int) const { return {}; }
  __device__ __forceinline__ NoConstants columns(int, int) const { return {}; }
  __device__ __forceinline__ void operator()(int m, int n, int N, Row, NoConstants, const v4f &v) const {
    if (m < rows0) store4(y0 + m * ld0, n, N, v, vec);
    else if (m >= split && m - split < rows0) store4(y1 + (m - split) * ld1, n, N, v, vec);
  }
};

// 64 x 64 blocks of 16-bit values, transposed through LDS.
constexpr int TRB = 64;
template <class E>
__device__ __forceinline__ void transposed_block(E (*t)[TRB + 2], E *out, int64_t ld, int r0, int c0, int rows, int cols) {
  __syncthreads();
  for (int i = threadIdx.x; i < TRB * TRB; i += 256) {
    const int c = i / TRB, r = i % TRB;  // out[c][r]
    if (c0 + c < cols && r0 + r < rows) out[(int64_t)(c0 + c) * ld + r0 + r] = t[r][c];
  }
}

// out[c][r] = in[r][c] for r below `rows`, zeros up to outCols; in has `cols` columns.
template <class E>
__global__ __launch_bounds__(256) void transpose_kernel(const E *in, int64_t ldi, int rows, int cols, E *out, int64_t ldo,
                                                        int outCols) {
  __shared__ E t[TRB][TRB + 2];
  const int r0 = blockIdx.y * TRB, c0 = blockIdx.x * TRB;
  for (int i = threadIdx.x; i < TRB * TRB; i += 256) {
    const int r = i / TRB, c = i % TRB;
    t[r][c] = r0 + r < rows && c0 + c < cols ? in[(int64_t)(r0 + r) * ldi + c0 + c] : (E)0.0f;
  }
  transposed_block(t, out, ldo, r0, c0, outCols, cols);
}

// Gradients of the projections, dG = dh * saved[0] and dU = dh * saved[1], side by side in rows of 2 Fp (zeros beside F),
// and the same transposed with zeros beside T.
template <class E>
__global__ __launch_bounds__(256) void gated_gradient_kernel(const E *dh, int64_t ldh, const float *saved, int64_t plane, int T,
                                                             int F, int Fp, int Tp, E *out, E *outT) {
  __shared__ E t[TRB][TRB + 2];
  const int r0 = blockIdx.y * TRB, c0 = blockIdx.x * TRB, which = blockIdx.z;
  for (int i = threadIdx.x; i < TRB * TRB; i += 256) {
    const int r = r0 + i / TRB, c = c0 + i % TRB;
    const E v = r < T && c < F ? (E)((float)dh[r * ldh + c] * saved[which * plane + (int64_t)r * F + c]) : (E)0.0f;
    t[i / TRB][i % TRB] = v;
    if (r < T && c < Fp) out[(int64_t)r * 2 * Fp + which * Fp + c] = v;
  }
  transposed_block(t, outT + (int64_t)which * Fp * Tp, Tp, r0, c0, Tp, Fp);
}

template <class E>
__global__ __launch_bounds__(256) void zero_rows_kernel(E *y, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < rows * cols; i += gridDim.x * 256ll) y[i / cols * ld + i % cols] = (E)0.0f;
}

inline bool half_type(int t) { return t == BNN_BF16 || t == BNN_F16; }
inline bool act_known(int a) { return a >= BNN_ACT_SILU && a <= BNN_ACT_RELU; }
inline int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }
constexpr int64_t MAX_DIM = (1 << 22) - 64;  // blocks of 64 rows within a launch's 65535; in bytes, doubled, 32 bits

template <int TY>
bnn_status gated_backward(const char *x, int64_t x_ld, const char *wg, int64_t wg_ld, const char *wu, int64_t wu_ld,
                          const float *saved, const void *dh_, int64_t dh_ld, int T, int D, int F, void *dx, int64_t dx_ld,
                          void *dwg, int64_t dwg_ld, void *dwu, int64_t dwu_ld, char *workspace, hipStream_t s) {
  using E = typename MmTraits<TY>::elem;
  const int Fp = (int)pad8(F), Tp = (int)pad8(T);
  E *grad = reinterpret_cast<E *>(workspace);              // [T, 2 Fp]
  E *gradT = grad + (int64_t)T * 2 * Fp;                   // [2 Fp, Tp]
  E *wT = gradT + (int64_t)2 * Fp * Tp;                    // [D, 2 Fp]
  E *xT = wT + (int64_t)D * 2 * Fp;                        // [D, Tp]
  const E *dh = static_cast<const E *>(dh_);
  const auto blocks = [](int64_t n) { return (uint32_t)((n + TRB - 1) / TRB); };
  {
    ProfScope ps(KID_GATED_GRADIENT, s);
    gated_gradient_kernel<E><<<dim3(blocks(Fp), blocks(Tp), 2), 256, 0, s>>>(dh, dh_ld, saved, (int64_t)T * F, T, F, Fp, Tp, grad, gradT);
  }
  {
    ProfScope ps(KID_TRANSPOSE, s);
    transpose_kernel<E><<<dim3(blocks(D), blocks(Fp)), 256, 0, s>>>(reinterpret_cast<const E *>(wg), wg_ld, F, D, wT, 2 * Fp, Fp);
    transpose_kernel<E><<<dim3(blocks(D), blocks(Fp)), 256, 0, s>>>(reinterpret_cast<const E *>(wu), wu_ld, F, D, wT + Fp, 2 * Fp, Fp);
    transpose_kernel<E><<<dim3(blocks(D), blocks(Tp)), 256, 0, s>>>(reinterpret_cast<const E *>(x), x_ld, T, D, xT, Tp, Tp);
  }
  if (bnn_status st = launch_status()) return st;
  MmOperands p = {};
  p.A = reinterpret_cast<const char *>(grad), p.lda = 4ll * Fp;
  p.B0 = p.B1 = reinterpret_cast<const char *>(wT), p.ldb0 = p.ldb1 = 4ll * Fp;
  p.M = T, p.N = D, p.kbytes = 4 * Fp;
  p.dma = mm_dma(p.A, p.lda) && mm_dma(p.B0, p.ldb0);
  const ProductEpilogue<E> ex = {static_cast<E *>(dx), nullptr, dx_ld, 0, T, T, rows_by(dx, dx_ld, 2, 4)};
  if (bnn_status st = run_product<TY, false>(p, ex, KID_GATED_FF_BACKWARD, KID_GATED_FF_BACKWARD, s)) return st;
  p.A = reinterpret_cast<const char *>(gradT), p.lda = 2ll * Tp;
  p.B0 = p.B1 = reinterpret_cast<const char *>(xT), p.ldb0 = p.ldb1 = 2ll * Tp;
  p.M = 2 * Fp, p.N = D, p.kbytes = 2 * Tp;
  p.dma = mm_dma(p.A, p.lda) && mm_dma(p.B0, p.ldb0);
  const ProductEpilogue<E> ew = {static_cast<E *>(dwg), static_cast<E *>(dwu), dwg_ld, dwu_ld, F, Fp,
                                 rows_by(dwg, dwg_ld, 2, 4) && rows_by(dwu, dwu_ld, 2, 4)};
  return run_product<TY, false>(p, ew, KID_GATED_FF_BACKWARD, KID_GATED_FF_BACKWARD, s);
}

// Gradients of an empty product.
template <class E>
void zero_rows(void *y, int64_t ld, int64_t rows, int64_t cols, hipStream_t s) {
  if (rows && cols) zero_rows_kernel<E><<<(uint32_t)std::min<int64_t>((rows * cols + 255) / 256, 4096), 256, 0, s>>>(static_cast<E *>(y), ld, rows, cols);
}

}  // namespace bnn

extern "C" size_t bnn_gated_ff_saved_bytes(int64_t T, int64_t F) {
  return T <= 0 || F <= 0 || T > bnn::MAX_DIM || F > bnn::MAX_DIM ? 0 : 8u * (size_t)T * (size_t)F;
}

extern "C" bnn_status bnn_gated_ff(const void *x, int64_t x_ld, const void *wg, int64_t wg_ld, const void *wu, int64_t wu_ld,
                                   int type, int64_t T, int64_t D, int64_t F, int act, void *h, int64_t h_ld, float *saved,
                                   void *stream) {
  using namespace bnn;
  if (T < 0 || F < 0 || D <= 0 || !float_type(type) || !act_known(act)) return BNN_ERR_SHAPE;
  if (x_ld < D || wg_ld < D || wu_ld < D || h_ld < F) return BNN_ERR_STRIDE;
  if (!half_type(type) || T > MAX_DIM || D > MAX_DIM || F > MAX_DIM) return BNN_ERR_UNSUPPORTED;
  if (T == 0 || F == 0) return BNN_OK;
  if (!x || !wg || !wu || !h) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned16(wg) || !aligned16(wu) || !aligned16(h) || !aligned16(saved)) return BNN_ERR_ALIGN;
  MmOperands p = {};
  p.A = static_cast<const char *>(x), p.lda = 2 * x_ld;
  p.B0 = static_cast<const char *>(wg), p.ldb0 = 2 * wg_ld;
  p.B1 = static_cast<const char *>(wu), p.ldb1 = 2 * wu_ld;
  p.M = (int)T, p.N = (int)F, p.kbytes = (int)(2 * D);
  p.dma = mm_dma(x, p.lda) && mm_dma(wg, p.ldb0) && mm_dma(wu, p.ldb1);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int vec = rows_by(h, h_ld, 2, 4), savedVec = F % 4 == 0;
  if (type == BNN_BF16)
    return run_product<MM_BF16, true>(p, GatedEpilogue<__bf16>{static_cast<__bf16 *>(h), h_ld, saved, T * F, act, vec, savedVec}, KID_GATED_FF, KID_GATED_FF, s);
  return run_product<MM_F16, true>(p, GatedEpilogue<_Float16>{static_cast<_Float16 *>(h), h_ld, saved, T * F, act, vec, savedVec}, KID_GATED_FF, KID_GATED_FF, s);
}

extern "C" bnn_status bnn_gated_ff_i8(const int8_t *x, int64_t x_ld, const float *x_scale, const int8_t *wg, int64_t wg_ld,
                                      const float *wg_scale, const int8_t *wu, int64_t wu_ld, const float *wu_scale, int64_t T,
                                      int64_t D, int64_t F, int act, void *h, int type, int64_t h_ld, void *stream) {
  using namespace bnn;
  if (T < 0 || F < 0 || D <= 0 || !float_type(type) || !act_known(act)) return BNN_ERR_SHAPE;
  if (x_ld < D || wg_ld < D || wu_ld < D || h_ld < F) return BNN_ERR_STRIDE;
  if (D > 131071 || T > MAX_DIM || F > MAX_DIM) return BNN_ERR_UNSUPPORTED;
  if (T == 0 || F == 0) return BNN_OK;
  if (!x || !x_scale || !wg || !wg_scale || !wu || !wu_scale || !h) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned16(x_scale) || !aligned16(wg) || !aligned16(wg_scale) || !aligned16(wu) || !aligned16(wu_scale) ||
      !aligned16(h))
    return BNN_ERR_ALIGN;
  MmOperands p = {};
  p.A = reinterpret_cast<const char *>(x), p.lda = x_ld;
  p.B0 = reinterpret_cast<const char *>(wg), p.ldb0 = wg_ld;
  p.B1 = reinterpret_cast<const char *>(wu), p.ldb1 = wu_ld;
  p.M = (int)T, p.N = (int)F, p.kbytes = (int)D;
  p.dma = mm_dma(x, x_ld) && mm_dma(wg, wg_ld) && mm_dma(wu, wu_ld);
  const GatedI8Epilogue epi = {x_scale, wg_scale, wu_scale, h, h_ld, type, act, rows_by(h, h_ld, float_size(type), 4)};
  return run_product<MM_I8, true>(p, epi, KID_GATED_FF_I8, KID_GATED_FF_I8, static_cast<hipStream_t>(stream));
}

extern "C" size_t bnn_gated_ff_backward_workspace_bytes(int64_t T, int64_t D, int64_t F) {
  using namespace bnn;
  if (T <= 0 || D <= 0 || F <= 0 || T > MAX_DIM || D > MAX_DIM || F > MAX_DIM) return 0;
  const size_t Fp = (size_t)pad8(F), Tp = (size_t)pad8(T);
  return 2 * (2 * Fp * (size_t)T + 2 * Fp * Tp + 2 * Fp * (size_t)D + Tp * (size_t)D);
}

extern "C" bnn_status bnn_gated_ff_backward(const void *x, int64_t x_ld, const void *wg, int64_t wg_ld, const void *wu,
                                            int64_t wu_ld, int type, int64_t T, int64_t D, int64_t F, const float *saved,
                                            const void *dh, int64_t dh_ld, void *dx, int64_t dx_ld, void *dwg, int64_t dwg_ld,
                                            void *dwu, int64_t dwu_ld, void *workspace, size_t workspace_bytes, void *stream) {
  using namespace bnn;
  if (T < 0 || F < 0 || D <= 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (x_ld < D || wg_ld < D || wu_ld < D || dh_ld < F || dx_ld < D || dwg_ld < D || dwu_ld < D) return BNN_ERR_STRIDE;
  if (!half_type(type) || T > MAX_DIM || D > MAX_DIM || F > MAX_DIM) return BNN_ERR_UNSUPPORTED;
  if ((T && !dx) || (F && (!dwg || !dwu))) return BNN_ERR_NULL;
  if (!aligned16(dx) || !aligned16(dwg) || !aligned16(dwu)) return BNN_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T == 0 || F == 0) {
    zero_rows<uint16_t>(dx, dx_ld, T, D, s);
    zero_rows<uint16_t>(dwg, dwg_ld, F, D, s);
    zero_rows<uint16_t>(dwu, dwu_ld, F, D, s);
    return T || F ? launch_status() : BNN_OK;
  }
  if (!x || !wg || !wu || !saved || !dh || !workspace) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned16(wg) || !aligned16(wu) || !aligned16(saved) || !aligned16(dh) || !aligned16(workspace))
    return BNN_ERR_ALIGN;
  if (workspace_bytes < bnn_gated_ff_backward_workspace_bytes(T, D, F)) return BNN_ERR_WORKSPACE;
  const auto run = type == BNN_BF16 ? gated_backward<MM_BF16> : gated_backward<MM_F16>;
  return run(static_cast<const char *>(x), x_ld, static_cast<const char *>(wg), wg_ld, static_cast<const char *>(wu), wu_ld, saved,
             dh, dh_ld, (int)T, (int)D, (int)F, dx, dx_ld, dwg, dwg_ld, dwu, dwu_ld, static_cast<char *>(workspace), s);
}
