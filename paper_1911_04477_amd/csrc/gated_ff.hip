// Gated feed-forward, h = act(x Wg^T) * (x Wu^T): both projections, the activation and the product in one kernel, from
// 16-bit floating-point operands (with its backward pass) or from 8-bit ones with scales.
#include <algorithm>
#include <cmath>

#include "bnn_testing.h"
#include "few_mm.h"
#include "kmajor_mm.h"
#include "rows.h"

namespace bnn {

// The normal distribution's function, and exp(-z^2 / 2).  Of a = |z| the tail is exp(-a^2 / 2) t P(t), t = 1 / (1 + 0.345 a): P is fitted
// to exp(a^2 / 2) (1 - erf(a / sqrt 2)) / 2 on 0 .. 14, least squares with weights moved to where the relative error is largest, 2e-8 at
// the end.  With what the squares and the exponent lose put back, a value below zero is off by 6 * 2^-24 of itself, as far as fp32's
// normal numbers reach (1 + erf there loses all of its digits).  Beyond 16 it is 0.  (fp16, 1000 x 1024 to 2321: 19.2 us, 18.7 with a
// formula good to 1.5e-7 of 1 and not of the value, 22.5 with erfcf.)
__device__ __forceinline__ float normal_function(float z, float &density) {
  constexpr float C = -0.72134752044448170f, C_REST = (float)(-0.72134752044448170368 - (double)C), LN2 = 0.69314718055994531f;
  const float a = fminf(fabsf(z), 16.0f);
  const float square = a * a, power = square * C;
  const float rest = fmaf(fmaf(a, a, -square), C, fmaf(square, C_REST, fmaf(square, C, -power)));
  const float t = __builtin_amdgcn_rcpf(fmaf(0.345f, a, 1.0f));
  density = __builtin_amdgcn_exp2f(power);
  density = fmaf(density, rest * LN2, density);
  float p = -0.028381976f;
  p = fmaf(p, t, 0.145282045f);
  p = fmaf(p, t, -0.271173209f);
  p = fmaf(p, t, 0.187196776f);
  p = fmaf(p, t, -0.0376017168f);
  p = fmaf(p, t, 0.111799605f);
  p = fmaf(p, t, 0.117238283f);
  p = fmaf(p, t, 0.138020888f);
  p = fmaf(p, t, 0.137619287f);
  const float tail = density * (t * p);
  return z < 0.0f ? tail : 1.0f - tail;
}

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
    float density;
    const float t = normal_function(z, density);
    a = z * t;
    if (SLOPE) slope = t + z * 0.39894228040143268f * density;
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

// f with the activation as a tag.
template <class F>
bnn_status with_act(int act, const F &f) {
  switch (act) {
    case BNN_ACT_SILU: return f(std::integral_constant<int, BNN_ACT_SILU>());
    case BNN_ACT_GELU: return f(std::integral_constant<int, BNN_ACT_GELU>());
    case BNN_ACT_GELU_TANH: return f(std::integral_constant<int, BNN_ACT_GELU_TANH>());
    default: return f(std::integral_constant<int, BNN_ACT_RELU>());
  }
}

// Where a backward pass will follow, `saved` takes what it multiplies the gradient of h with, in fp32 (16 bits would round
// the gradients of the projections twice): act'(g) * u for that of g = x Wg^T, act(g) for that of u = x Wu^T.
// ACT, SAVE: known when the kernel is compiled, or -1; then they are looked at for every group of columns.
template <class E, int ACT = -1, int SAVE = -1>
struct GatedEpilogue {
  E *h;
  int64_t ldh;
  float *saved;
  int64_t plane;  // values in one of the two
  int act;
  using Row = NoConstants;
  __device__ __forceinline__ Row row(int) const { return {}; }
  __device__ __forceinline__ NoConstants columns(int, int) const { return {}; }
  __device__ __forceinline__ void operator()(int m, int n, int N, Row, NoConstants, const v4f &g, const v4f &u) const {
    float o[4], dg[4], du[4];
    const int act = ACT < 0 ? this->act : ACT;
    if (SAVE < 0 ? saved != nullptr : SAVE) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float slope;
        du[i] = activation<true>(act, g[i], slope);
        dg[i] = slope * u[i];
        o[i] = du[i] * u[i];
      }
      store4(saved + (int64_t)m * N, n, N, dg);
      store4(saved + plane + (int64_t)m * N, n, N, du);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float none;
        o[i] = activation<false>(act, g[i], none) * u[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("" : "+v"(o[i]));  // h rounds the fp32 product in every form: no product and conversion in one
    store4(h + m * ldh, n, N, o);
  }
  template <class F>
  bnn_status fixed(const F &f) const {
    return with_act(act, [&](auto a) {
      constexpr int A = decltype(a)::value;
      return saved ? f(GatedEpilogue<E, A, 1>{h, ldh, saved, plane, act}) : f(GatedEpilogue<E, A, 0>{h, ldh, saved, plane, act});
    });
  }
};

template <int ACT = -1>
struct GatedI8Epilogue {
  const float *sx, *sg, *su;
  void *h;
  int64_t ldh;
  int type, act;
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
      o[i] = activation<false>(ACT < 0 ? act : ACT, (float)g[i] * a * c.g[i], none) * ((float)u[i] * a * c.u[i]);
    }
    if (type == BNN_BF16) store4(static_cast<__bf16 *>(h) + m * ldh, n, N, o);
    else if (type == BNN_F16) store4(static_cast<_Float16 *>(h) + m * ldh, n, N, o);
    else store4(static_cast<float *>(h) + m * ldh, n, N, o);
  }
  template <class F>
  bnn_status fixed(const F &f) const {
    return with_act(act, [&](auto a) { return f(GatedI8Epilogue<decltype(a)::value>{sx, sg, su, h, ldh, type, act}); });
  }
};

// A product rounded to the operands' type; rows from `split` on go to a second matrix.  part: sums of a share of k go there
// instead, in fp32, [shares][M][ld].
template <class E>
struct ProductEpilogue {
  E *y0, *y1;
  int64_t ld0, ld1;
  int rows0, split;  // rows0 <= split: rows between them are padding
  int D;             // columns that are stored
  float *part;
  int64_t plane, part_ld;
  const float *range;  // fp16: what a sum is multiplied with (gated_gradient_scale_kernel)
  __device__ __forceinline__ float factor() const {
    if constexpr (std::is_same<E, _Float16>::value) return *range;
    return 1.0f;
  }
  __device__ __forceinline__ void store(int m, int n, v4f v, float factor) const {
    if constexpr (std::is_same<E, _Float16>::value) v *= factor;
    if (m < rows0) store4(y0 + m * ld0, n, D, v);
    else if (m >= split && m - split < rows0) store4(y1 + (m - split) * ld1, n, D, v);
  }
  __device__ __forceinline__ void operator()(int m, int n, int, int share, float factor, const v4f &v) const {
    if (part) *reinterpret_cast<v4f *>(part + share * plane + m * part_ld + n) = v;
    else store(m, n, v, factor);
  }
};

template <class E>
__global__ __launch_bounds__(256) void product_sums_kernel(ProductEpilogue<E> epi, int M, int shares) {
  const int64_t quads = epi.part_ld / 4, i = wide_block() * 256 + threadIdx.x;
  if (i >= M * quads) return;
  const int m = (int)(i / quads), n = (int)(i - m * quads) * 4;
  v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < shares; ++s) sum += *reinterpret_cast<const v4f *>(epi.part + s * epi.plane + m * epi.part_ld + n);
  if (n < epi.D) epi.store(m, n, sum, epi.factor());
}

// Gradients of the projections, dG = dh * saved[0] and dU = dh * saved[1], side by side in rows of 2 Fp (zeros beside F):
// eight values a thread.  Bound by memory (14 B a value; 8192 x 8192 160 to 170 us again and again, 5.6 TB/s, 200 to 220 right after the
// forward pass).
// They are rounded to the operands' type, the one rounding on the way from dh to the results: the matrix units multiply
// 16-bit values, and each gradient as a sum of two of them would double the products.  It adds as much to a result's error as
// the result's own rounding does: 1.4 times that of a pass with fp32 operands, in the 2-norm.
template <class E>
struct GradientOf {
  const E *dh;
  int64_t ldh;
  const float *saved;
  int64_t plane, groups;
  int F, Fp;
  E *out;
  // Group i, times `scale`; returns the largest finite magnitude before that, as bits.
  __device__ __forceinline__ uint32_t write(int64_t i, float scale) const {
    const int per = Fp / 8;
    const int64_t r = i / per;
    const int c = (int)(i - r * per) * 8;
    float d[8], g[8], u[8];
    load8(d, dh + r * ldh, c, F);
    load8(g, saved + r * F, c, F);
    load8(u, saved + plane + r * F, c, F);
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[j] *= d[j], u[j] *= d[j];
      if constexpr (std::is_same<E, _Float16>::value) {
        const uint32_t a = magnitude(g[j]), b = magnitude(u[j]);
        top = max(top, max(a < 0x7f800000u ? a : 0u, b < 0x7f800000u ? b : 0u));
        g[j] *= scale, u[j] *= scale;
      }
    }
    store8(out + r * 2 * Fp, c, Fp, g);
    store8(out + r * 2 * Fp + Fp, c, Fp, u);
    return top;
  }
};
template <class E>
__global__ __launch_bounds__(256) void gated_gradient_kernel(GradientOf<E> q) {
  const int64_t i = wide_block() * 256 + threadIdx.x;
  if (i < q.groups) q.write(i, 1.0f);
}

// fp16 holds less than the products dh * saved can be: they pass 65504 where the results do not, and what lies below 2^-14 loses
// bits that sums over many rows or columns still need.  So all of them are multiplied with one power of two, and the sums
// of products with its inverse: 1 where the largest (finite) magnitude is in 1 .. 65504, when what is lost below 2^-14
// is at most 2^-25 of it, else what brings it to 2^14 .. 2^15.  The first kernel writes them as they are, with the largest of every
// workgroup; the second writes them again only where the scale is not 1.  (Backward of 1000 x 1024 to 2321 54.7 -> 57.3 us where it is
// 1, 63 where not; 8192 x 4096 to 8192 1 and 10 % longer.)
constexpr int GRADIENT_THREADS = 256, SCALE_THREADS = 1024, SCALE_BLOCKS = 256;
__device__ __forceinline__ float range_scale(uint32_t top) {
  if (top == 0u || (top >= 0x3f800000u && top <= 0x477fe000u)) return 1.0f;
  const int e = 14 - ((int)(top >> 23) - 127);  // to [2^14, 2^15), as far as both powers are normal numbers
  return __uint_as_float((uint32_t)(127 + max(-126, min(126, e))) << 23);
}
__global__ __launch_bounds__(GRADIENT_THREADS) void gated_gradient_top_kernel(GradientOf<_Float16> q, uint32_t *tops) {
  __shared__ uint32_t lds[16];
  const int64_t i = wide_block() * GRADIENT_THREADS + threadIdx.x;
  uint32_t top = i < q.groups ? q.write(i, 1.0f) : 0u;
  top = wave_reduce(top, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0 && i < q.groups) tops[wide_block()] = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
}
// Every workgroup takes the largest of all (8192 x 8192: 128 KB of them), and its share of the groups where they are written again.
__global__ __launch_bounds__(SCALE_THREADS) void gated_gradient_scale_kernel(GradientOf<_Float16> q, const uint32_t *tops, int64_t n, float *factor) {
  __shared__ uint32_t lds[16];
  clear_words(lds);
  uint32_t top = 0u;
  for (int64_t k = threadIdx.x; k < n; k += SCALE_THREADS) top = max(top, tops[k]);
  const float scale = range_scale(__float_as_uint(team_max_magnitude<true>(top, lds)));
  if (blockIdx.x == 0 && threadIdx.x == 0) *factor = 1.0f / scale;
  if (scale == 1.0f) return;
  for (int64_t i = blockIdx.x * (int64_t)SCALE_THREADS + threadIdx.x; i < q.groups; i += gridDim.x * (int64_t)SCALE_THREADS) q.write(i, scale);
}

// Rows of D values as rows of Dp that start on 16 bytes, zeros behind them.
template <class E>
__global__ __launch_bounds__(256) void realign_kernel(const E *in, int64_t ld, int64_t groups, int D, int Dp, E *out) {
  const int64_t i = wide_block() * 256 + threadIdx.x;
  if (i >= groups) return;
  const int per = Dp / 8;
  const int64_t r = i / per;
  const int c = (int)(i - r * per) * 8;
  float v[8];
  load8(v, in + r * ld, c, D);
  store8(out + r * Dp, c, Dp, v);
}

template <class E>
__global__ __launch_bounds__(256) void zero_rows_kernel(E *y, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < rows * cols; i += gridDim.x * 256ll) y[i / cols * ld + i % cols] = (E)0.0f;
}

inline bool half_type(int t) { return t == BNN_BF16 || t == BNN_F16; }
inline bool act_known(int a) { return a >= BNN_ACT_SILU && a <= BNN_ACT_RELU; }
inline int64_t pad(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
constexpr int64_t MAX_DIM = (1 << 22) - 64;  // km_at: 255 rows of two projections' gradients within 32 bits

// Which kernel takes a k-major product, and into how many shares its k is split: the cheapest by microseconds a step and a
// round of tiles, what a round costs beside its steps, and the shares' way through memory.  Measured in bf16: 256 x 256
// tiles 8192 x 4096 by k 16384 799 us, 16384 x 4096 by k 256 72; 128 x 128 with one tile a unit 256 x 4096 by k 16384 in
// four shares 39, 1000 x 1024 by k 4642 in four 18; two a unit 1040 and 62; 64 x 64 one a unit 30 (1000 x 1024), two 101.
struct KmPlan {
  int form, shares;
};
inline KmPlan km_plan(int64_t M, int64_t N, int64_t steps) {
  constexpr struct {
    int tile, slots;
    double step, round;
  } forms[] = {{256, 256, 1.5, 11.5}, {128, 256, 0.6, 4.0}, {128, 512, 1.016, 3.6}, {64, 256, 0.4, 1.5}, {64, 512, 0.55, 1.5}};
  KmPlan best = {0, 1};
  double least = 1e300;
  for (int f = 0; f < 5; ++f)
    for (int shares = 1; shares <= 32 && (shares == 1 || shares * 4 <= steps); ++shares) {
      const double tiles = (double)((M - 1) / forms[f].tile + 1) * (double)((N - 1) / forms[f].tile + 1) * shares;
      if (f % 2 && tiles > forms[f].slots) continue;  // one tile a unit
      const double rounds = std::ceil(tiles / forms[f].slots);
      const double cost = rounds * ((steps + shares - 1) / shares * forms[f].step + forms[f].round) +
                          (shares > 1 ? 4.0 + 8e-6 / 4.0 * shares * (double)M * (double)N : 0.0);
      if (cost < least) least = cost, best = {f, shares};
    }
  return best;
}

// The parts of the backward pass's workspace, in bytes from its start.
struct GatedSpace {
  int64_t Fp, Dp, wg, wu, x, range, part, end;
};
inline GatedSpace gated_space(int64_t T, int64_t D, int64_t F) {
  GatedSpace g;
  g.Fp = pad(F, KM_STEP), g.Dp = pad(D, 8);
  g.wg = pad(T * 2 * g.Fp * 2, 256);  // gradients of the projections before it
  g.wu = g.wg + pad(F * g.Dp * 2, 256);
  g.x = g.wu + pad(F * g.Dp * 2, 256);
  g.range = g.x + pad(T * g.Dp * 2, 256);
  g.part = g.range + 256 + pad((T * g.Fp / 8 / GRADIENT_THREADS + 1) * 4, 256);  // the factor, the workgroups' largest
  const KmPlan x = km_plan(T, g.Dp, 2 * (F / KM_STEP)), w = km_plan(2 * g.Fp, g.Dp, T / KM_STEP);
  g.end = g.part + 4 * std::max(x.shares > 1 ? x.shares * T * g.Dp : 0, w.shares > 1 ? w.shares * 2 * g.Fp * g.Dp : 0);
  return g;
}

template <int TY, bool A_ROWS, class E>
bnn_status km_product(KmOperands p, ProductEpilogue<E> epi, float *part, hipStream_t s) {
  const KmPlan plan = km_plan(p.M, p.N, (int64_t)p.K / KM_STEP * p.segments);
  p.splits = plan.shares;
  if (plan.shares > 1) epi.part = part, epi.part_ld = p.N, epi.plane = (int64_t)p.M * p.N;
  bnn_status st;
  switch (plan.form) {
    case 0: st = launch_km_tile<TY, 256, 256, 2, 2, 2, A_ROWS>(p, epi, KID_GATED_FF_BACKWARD, s); break;
    case 1: st = launch_km_tile<TY, 128, 128, 2, 4, 4, A_ROWS>(p, epi, KID_GATED_FF_BACKWARD, s); break;
    case 2: st = launch_km_tile<TY, 128, 128, 2, 2, 2, A_ROWS>(p, epi, KID_GATED_FF_BACKWARD, s); break;
    default: st = launch_km_tile<TY, 64, 64, 2, 2, 4, A_ROWS>(p, epi, KID_GATED_FF_BACKWARD, s);
  }
  if (st || plan.shares == 1) return st;
  ProfScope ps(KID_PRODUCT_SUMS, s);
  product_sums_kernel<E><<<wide_grid(((int64_t)p.M * p.N / 4 + 255) / 256), 256, 0, s>>>(epi, p.M, plan.shares);
  return launch_status();
}

template <int TY>
bnn_status gated_backward(const char *x, int64_t x_ld, const char *wg, int64_t wg_ld, const char *wu, int64_t wu_ld,
                          const float *saved, const void *dh, int64_t dh_ld, int T, int D, int F, void *dx, int64_t dx_ld,
                          void *dwg, int64_t dwg_ld, void *dwu, int64_t dwu_ld, char *workspace, hipStream_t s) {
  using E = typename MmTraits<TY>::elem;
  const GatedSpace g = gated_space(T, D, F);
  const int Fp = (int)g.Fp, Dp = (int)g.Dp;
  E *const grad = reinterpret_cast<E *>(workspace);
  float *const part = reinterpret_cast<float *>(workspace + g.part);
  float *const factor = reinterpret_cast<float *>(workspace + g.range);
  const auto blocks = [](int64_t n) { return (n + 255) / 256; };
  {
    const GradientOf<E> q = {static_cast<const E *>(dh), dh_ld, saved, (int64_t)T * F, (int64_t)T * Fp / 8, F, Fp, grad};
    if constexpr (TY == MM_F16) {
      uint32_t *const tops = reinterpret_cast<uint32_t *>(workspace + g.range + 256);
      const int64_t grid = blocks(q.groups);
      {
        ProfScope ps(KID_GATED_GRADIENT, s);
        gated_gradient_top_kernel<<<wide_grid(grid), GRADIENT_THREADS, 0, s>>>(q, tops);
      }
      ProfScope ps(KID_GATED_GRADIENT, s);
      gated_gradient_scale_kernel<<<(uint32_t)std::min<int64_t>(grid, SCALE_BLOCKS), SCALE_THREADS, 0, s>>>(q, tops, grid, factor);
    } else {
      ProfScope ps(KID_GATED_GRADIENT, s);
      gated_gradient_kernel<E><<<wide_grid(blocks(q.groups)), 256, 0, s>>>(q);
    }
  }
  // the products take columns eight at a time, from rows that start on 16 bytes
  const auto fits = [&](const char *m, int64_t ld) { return D == Dp && mm_dma(m, 2 * ld); };
  const auto realign = [&](const char *&m, int64_t &ld, int64_t rows, int64_t at) {
    const int64_t n = rows * Dp / 8;
    ProfScope ps(KID_REALIGN, s);
    realign_kernel<E><<<wide_grid(blocks(n)), 256, 0, s>>>(reinterpret_cast<const E *>(m), ld, n, D, Dp, reinterpret_cast<E *>(workspace + at));
    m = workspace + at, ld = Dp;
  };
  const bool as_they_are = fits(wg, wg_ld) && fits(wu, wu_ld) && wg_ld == wu_ld;  // one row stride for both
  if (!as_they_are) realign(wg, wg_ld, F, g.wg), realign(wu, wu_ld, F, g.wu);
  if (!fits(x, x_ld)) realign(x, x_ld, T, g.x);
  if (bnn_status st = launch_status()) return st;
  KmOperands p = {};
  p.A = workspace, p.lda = 4ll * Fp, p.segA = Fp;
  p.B0 = wg, p.B1 = wu, p.ldb = 2 * wg_ld;
  p.M = T, p.N = Dp, p.K = F, p.segments = 2;
  ProductEpilogue<E> epi = {static_cast<E *>(dx), nullptr, dx_ld, 0, T, T, D, nullptr, 0, 0, factor};
  if (bnn_status st = km_product<TY, true>(p, epi, part, s)) return st;
  p.B0 = p.B1 = x, p.ldb = 2 * x_ld, p.segA = 0;
  p.M = 2 * Fp, p.K = T, p.segments = 1;
  epi = {static_cast<E *>(dwg), static_cast<E *>(dwu), dwg_ld, dwu_ld, F, Fp, D, nullptr, 0, 0, factor};
  return km_product<TY, false>(p, epi, part, s);
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
  if (type == BNN_BF16)
    return run_product<MM_BF16, true>(p, GatedEpilogue<__bf16>{static_cast<__bf16 *>(h), h_ld, saved, T * F, act}, KID_GATED_FF, KID_GATED_FF, s);
  return run_product<MM_F16, true>(p, GatedEpilogue<_Float16>{static_cast<_Float16 *>(h), h_ld, saved, T * F, act}, KID_GATED_FF, KID_GATED_FF, s);
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
  const GatedI8Epilogue<> epi = {x_scale, wg_scale, wu_scale, h, h_ld, type, act};
  return run_product<MM_I8, true>(p, epi, KID_GATED_FF_I8, KID_GATED_FF_I8, static_cast<hipStream_t>(stream));
}

extern "C" size_t bnn_gated_ff_backward_workspace_bytes(int64_t T, int64_t D, int64_t F) {
  using namespace bnn;
  if (T <= 0 || D <= 0 || F <= 0 || T > MAX_DIM || D > MAX_DIM || F > MAX_DIM) return 0;
  return (size_t)gated_space(T, D, F).end;
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

extern "C" int bnn_testing_product_form(int64_t M, int64_t N, int weights, int aligned, int units) {
  if (M <= 0 || N <= 0 || M > INT32_MAX - 256 || N > INT32_MAX - 256 || weights < 1 || weights > 2 || units < 1) return -1;
  return bnn::mm_form((int)M, (int)N, weights == 2, aligned != 0, units);
}

extern "C" int bnn_testing_gated_backward_plan(int64_t T, int64_t D, int64_t F, int64_t *values) {
  using namespace bnn;
  if (T <= 0 || D <= 0 || F <= 0 || T > MAX_DIM || D > MAX_DIM || F > MAX_DIM || !values) return -1;
  const GatedSpace g = gated_space(T, D, F);
  const KmPlan x = km_plan(T, g.Dp, 2 * (F / KM_STEP)), w = km_plan(2 * g.Fp, g.Dp, T / KM_STEP);
  constexpr int tile[] = {256, 128, 128, 64, 64};
  values[0] = x.form, values[1] = x.shares, values[2] = w.form, values[3] = w.shares;
  values[4] = km_at(std::min<int64_t>(tile[x.form], T) - 1, 4 * g.Fp, 7 * 16);
  return 0;
}
