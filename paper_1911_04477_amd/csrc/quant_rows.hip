// Rows of floating-point values as 8-bit integers with one scale a row (bnn_quant_rows_i8).
#include "rows.h"

namespace bnn {

struct QuantParams {
  const void *x;
  int64_t x_ld, q_ld;
  int8_t *q;
  float *scale;
  int64_t rows;
  int K;
};

// A row a wave (four of them a workgroup), or (BLOCK) a row a workgroup; NV pieces of eight values a thread, held in
// registers between the maximum and the rounding.  NV 0: rows of any length, read twice.  Bound by memory (8192 x 4096
// bf16 17 to 20 us, 5.0 to 5.9 TB/s).
template <class E, bool BLOCK, int MAXT, int NV, int EDGE>
__global__ __launch_bounds__(MAXT) void quant_rows_kernel(QuantParams p) {
  __shared__ uint32_t lds[16];
  if constexpr (BLOCK) clear_words(lds);
  const int T = BLOCK ? blockDim.x : 64, t = BLOCK ? threadIdx.x : threadIdx.x & 63;
  const int64_t row = BLOCK ? wide_block() : wide_block() * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;  // whole workgroups, or whole waves of those without barriers
  const E *x = static_cast<const E *>(p.x) + row * p.x_ld;
  int8_t *q = p.q + row * p.q_ld;
  uint32_t top = 0u;
  if constexpr (NV > 0) {
    Piece8<E> w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) w[i].load(x, Place8<EDGE>((i * T + t) * 8, p.K), p.K);
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place8<EDGE> at((i * T + t) * 8, p.K);
      if (at.shift) w[i].settle(at);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (float)w[i].v[j], top = max(top, magnitude(v[i][j]));
    }
    const RowScale s = row_scale(team_max_magnitude<BLOCK>(top, lds));
#pragma unroll
    for (int i = 0; i < NV; ++i) store_q8(q, (i * T + t) * 8, p.K, v[i], s.inv);
    if (t == 0) p.scale[row] = s.scale;
  } else {
    for (int c = t * 8; c < p.K; c += T * 8) {
      float v[8];
      load8(v, x, c, p.K);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[j]));
    }
    const RowScale s = row_scale(team_max_magnitude<BLOCK>(top, lds));
    for (int c = t * 8; c < p.K; c += T * 8) {
      float v[8];
      load8(v, x, c, p.K);
      store_q8(q, c, p.K, v, s.inv);
    }
    if (t == 0) p.scale[row] = s.scale;
  }
}

}  // namespace bnn

extern "C" bnn_status bnn_quant_rows_i8(const void *x, int type, int64_t rows, int64_t K, int64_t x_ld, int8_t *q,
                                        int64_t q_ld, float *scale, void *stream) {
  using namespace bnn;
  if (rows < 0 || K <= 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (x_ld < K || q_ld < K) return BNN_ERR_STRIDE;
  if (K > (1 << 28) || rows > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  if (rows == 0) return BNN_OK;
  if (!x || !q || !scale) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned16(q) || !aligned16(scale)) return BNN_ERR_ALIGN;
  const QuantParams p = {x, x_ld, q_ld, q, scale, rows, (int)K};
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_QUANT_ROWS, s);
  with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    const auto run = [&](auto whole, auto ragged, int block, int teams) {
      (row_edge(K) == EDGE_WHOLE ? whole : ragged)<<<wide_grid((rows - 1) / teams + 1), block, 0, s>>>(p);
    };
#define BNN_FORMS(...) quant_rows_kernel<E, __VA_ARGS__, EDGE_WHOLE>, quant_rows_kernel<E, __VA_ARGS__, EDGE_RAGGED>
    if (K < 8) quant_rows_kernel<E, false, 256, 1, EDGE_SMALL><<<wide_grid((rows - 1) / 4 + 1), 256, 0, s>>>(p);
    else if (K <= 512) run(BNN_FORMS(false, 256, 1), 256, 4);
    else if (K <= 4096) run(BNN_FORMS(true, 512, 1), row_threads(K, 1), 1);
    else if (K <= 32768) run(BNN_FORMS(true, 1024, 4), row_threads(K, 4), 1);
    else quant_rows_kernel<E, true, 1024, 0, EDGE_RAGGED><<<wide_grid(rows), 1024, 0, s>>>(p);
#undef BNN_FORMS
  });
  return launch_status();
}
