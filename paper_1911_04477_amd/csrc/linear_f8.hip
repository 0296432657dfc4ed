// Products of e4m3 matrices with block scales: the linear layer (bnn_linear_f8), the same for rows sorted by expert with a
// weight for each (bnn_expert_linear_f8), and the gradients of such weights (bnn_expert_linear_f8_dw).
#include <algorithm>

#include "bnn_testing.h"
#include "f8_mm.h"
#include "few_mm.h"

namespace bnn {

// Which kernel takes a product, by rounds of tiles as in few_mm.h.  rows: of a group, on average, and groups: how many.
enum : int { F8_256, F8_128, F8_64, F8_32, F8_FORM_COUNT, F8_FEW = 8 };
constexpr MmForm F8_FORMS[F8_FORM_COUNT] = {{256, 256, 100, 200}, {128, 128, 45, 74}, {64, 64, 22, 32}, {32, 64, 17, 24}};
inline int f8_form(int64_t rows, int64_t groups, int64_t N, bool small, int64_t units) {
  if (rows <= 16) return F8_FEW;
  int best = F8_64;
  int64_t least = INT64_MAX;
  for (int f = small ? F8_128 : F8_256; f < F8_FORM_COUNT; ++f) {
    const MmForm &t = F8_FORMS[f];
    const int64_t tiles = groups * ((rows - 1) / t.bm + 1) * ((N - 1) / t.bn + 1);
    const int64_t cost = t.bm == 256 ? (tiles + units - 1) / units * t.one : tiles <= units ? t.one : (tiles + 2 * units - 1) / (2 * units) * t.two;
    if (cost <= least) least = cost, best = f;
  }
  return best;
}

template <int BM, int BN, int WGM, int WGN, int STAGES, bool WIDE, bool EXACT>
bnn_status launch_f8_tile(F8Operands p, hipStream_t s) {
  p.tilesN = (p.N - 1) / BN + 1;
  // groups of rows: each has a part of a tile more than its rows fill at most
  p.tilesM = p.groups == F8_GROUP_ROWS ? p.M / BM + std::min(p.E, p.M) : (p.M - 1) / BM + 1;
  const int64_t tiles = (int64_t)p.tilesM * p.tilesN * (p.groups == F8_GROUP_K ? p.E : 1);
  if ((int64_t)p.tilesM * p.tilesN > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  ProfScope ps(KID_LINEAR_F8, s);
  wide_launches(tiles, [&](int64_t first, uint32_t n) {
    p.first = first;
    f8_tile_kernel<BM, BN, WGM, WGN, STAGES, WIDE, EXACT><<<n, 64 * WGM * WGN, 0, s>>>(p);
  });
  return launch_status();
}

template <bool WIDE>
bnn_status launch_f8_few(F8Operands p, hipStream_t s) {
  p.tilesN = (p.N - 1) / 16 + 1;
  p.tilesM = p.groups == F8_GROUP_ROWS ? p.M / 16 + std::min(p.E, p.M) : (p.M - 1) / 16 + 1;
  if ((int64_t)p.tilesM * p.tilesN > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  ProfScope ps(KID_LINEAR_F8_FEW, s);
  wide_launches((int64_t)p.tilesM * p.tilesN * (p.groups == F8_GROUP_K ? p.E : 1), [&](int64_t first, uint32_t n) {
    p.first = first;
    f8_few_kernel<8, WIDE><<<n, 512, 0, s>>>(p);
  });
  return launch_status();
}

template <bool WIDE, bool EXACT>
bnn_status run_f8_as(const F8Operands &p, hipStream_t s) {
  int64_t rows = p.M, groups = 1;
  if (p.groups == F8_GROUP_ROWS) groups = std::min(p.E, p.M), rows = (p.M - 1) / groups + 1;
  if (p.groups == F8_GROUP_K) groups = p.E;
  switch (f8_form(rows, groups, p.N, WIDE, device_cu_count())) {
    case F8_256:
      if constexpr (!WIDE) return launch_f8_tile<256, 256, 2, 2, 2, false, EXACT>(p, s);
    case F8_128: return launch_f8_tile<128, 128, 2, 2, 2, WIDE, EXACT>(p, s);
    case F8_64: return launch_f8_tile<64, 64, 2, 2, 3, WIDE, EXACT>(p, s);
    case F8_32: return launch_f8_tile<32, 64, 1, 2, 4, WIDE, EXACT>(p, s);
    default: return launch_f8_few<WIDE>(p, s);
  }
}
template <bool WIDE>
bnn_status run_f8(const F8Operands &p, hipStream_t s) {
  return p.type == BNN_F32 ? run_f8_as<WIDE, true>(p, s) : run_f8_as<WIDE, false>(p, s);
}

// B's scales, checked: N rows of K values, of which `per` share a row of scales.
bnn_status f8_weight(F8Operands &p, const uint8_t *b, int64_t ldb, const void *scale, int scale_type, int64_t scale_ld, int per, int64_t N,
                     int64_t K) {
  if (scale_type != BNN_SCALE_E8M0 && scale_type != BNN_SCALE_F32) return BNN_ERR_SHAPE;
  if (per != F8_BLOCK && (per != 1 || scale_type == BNN_SCALE_F32)) return BNN_ERR_SHAPE;
  if (scale_type == BNN_SCALE_F32) {
    if (scale_ld < f8_blocks(K)) return BNN_ERR_STRIDE;
    const bnn_status st = f8_check(b, ldb, scale, f8_scale_bytes(K), K);
    if (st != BNN_OK) return st;
  } else {
    const bnn_status st = f8_check(b, ldb, scale, scale_ld, K);
    if (st != BNN_OK) return st;
  }
  p.B = reinterpret_cast<const char *>(b), p.ldb = ldb, p.sb = scale, p.sb_ld = scale_ld, p.sb_shift = per == 1 ? 0 : 7;
  p.N = (int)N;
  return BNN_OK;
}

constexpr int64_t F8_MOST = INT32_MAX - 256;

}  // namespace bnn

extern "C" bnn_status bnn_linear_f8(const uint8_t *a, int64_t lda, const uint8_t *a_scale, int64_t a_scale_ld, const uint8_t *b,
                                    int64_t ldb, const void *b_scale, int b_scale_type, int64_t b_scale_ld, int b_scale_rows,
                                    const float *bias, int64_t M, int64_t N, int64_t K, void *y, int type, int64_t ldy,
                                    void *stream) {
  using namespace bnn;
  if (M < 0 || N < 0 || K <= 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (ldy < N) return BNN_ERR_STRIDE;
  if (M > F8_MOST || N > F8_MOST || K > (1 << 22)) return BNN_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return BNN_OK;
  F8Operands p = {};
  bnn_status st = f8_check(a, lda, a_scale, a_scale_ld, K);
  if (st == BNN_OK) st = f8_weight(p, b, ldb, b_scale, b_scale_type, b_scale_ld, b_scale_rows, N, K);
  if (st != BNN_OK) return st;
  if (!y) return BNN_ERR_NULL;
  if (!aligned16(y) || !aligned16(bias)) return BNN_ERR_ALIGN;
  p.A = reinterpret_cast<const char *>(a), p.lda = lda, p.sa = a_scale, p.sa_ld = a_scale_ld;
  p.M = (int)M, p.blocks = (int)f8_blocks(K), p.bias = bias, p.y = y, p.type = type, p.ldy = ldy;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return b_scale_type == BNN_SCALE_F32 ? run_f8<true>(p, s) : run_f8<false>(p, s);
}

extern "C" bnn_status bnn_expert_linear_f8(const uint8_t *a, int64_t lda, const uint8_t *a_scale, int64_t a_scale_ld,
                                           const int32_t *offsets, int64_t experts, const uint8_t *b, int64_t ldb, int64_t b_expert_ld,
                                           const void *b_scale, int b_scale_type, int64_t b_scale_ld, int64_t b_scale_expert_ld,
                                           int b_scale_rows, int64_t S, int64_t N, int64_t K, void *y, int type, int64_t ldy,
                                           void *stream) {
  using namespace bnn;
  if (S < 0 || N < 0 || K <= 0 || experts < 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (ldy < N) return BNN_ERR_STRIDE;
  if (S > F8_MOST || N > F8_MOST || K > (1 << 22) || experts > 65535) return BNN_ERR_UNSUPPORTED;
  if (S == 0 || N == 0 || experts == 0) return BNN_OK;
  F8Operands p = {};
  bnn_status st = f8_check(a, lda, a_scale, a_scale_ld, K);
  if (st == BNN_OK) st = f8_weight(p, b, ldb, b_scale, b_scale_type, b_scale_ld, b_scale_rows, N, K);
  if (st != BNN_OK) return st;
  const int64_t scale_rows = b_scale_rows == 1 ? N : f8_blocks(N);
  if (experts > 1 && (b_expert_ld / N < ldb || b_expert_ld % 16 || b_scale_expert_ld / scale_rows < b_scale_ld || (b_scale_type == BNN_SCALE_E8M0 && b_scale_expert_ld % 4)))
    return BNN_ERR_STRIDE;
  if (!offsets || !y) return BNN_ERR_NULL;
  if (!aligned16(offsets) || !aligned16(y)) return BNN_ERR_ALIGN;
  p.A = reinterpret_cast<const char *>(a), p.lda = lda, p.sa = a_scale, p.sa_ld = a_scale_ld;
  p.M = (int)S, p.blocks = (int)f8_blocks(K), p.y = y, p.type = type, p.ldy = ldy;
  p.groups = F8_GROUP_ROWS, p.offsets = offsets, p.E = (int)experts, p.b_es = b_expert_ld;
  p.sb_es = b_scale_expert_ld * (b_scale_type == BNN_SCALE_F32 ? 4 : 1);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return b_scale_type == BNN_SCALE_F32 ? run_f8<true>(p, s) : run_f8<false>(p, s);
}

extern "C" bnn_status bnn_expert_linear_f8_dw(const uint8_t *a, int64_t lda, const uint8_t *a_scale, int64_t a_scale_ld,
                                              const uint8_t *b, int64_t ldb, const uint8_t *b_scale, int64_t b_scale_ld,
                                              const int32_t *offsets, int64_t experts, int64_t N, int64_t K, int64_t S, void *dw,
                                              int type, int64_t dw_ld, int64_t dw_expert_ld, void *stream) {
  using namespace bnn;
  if (S < 0 || N < 0 || K < 0 || experts < 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (dw_ld < K || (experts > 1 && N > 0 && dw_expert_ld / N < dw_ld)) return BNN_ERR_STRIDE;
  if (S > (1 << 22) - F8_BLOCK || N > F8_MOST || K > F8_MOST || experts > 65535) return BNN_ERR_UNSUPPORTED;
  if (N == 0 || K == 0 || experts == 0) return BNN_OK;
  F8Operands p = {};
  if (S > 0) {  // else every group is empty, and the result 0
    bnn_status st = f8_check(a, lda, a_scale, a_scale_ld, S);
    if (st == BNN_OK) st = f8_weight(p, b, ldb, b_scale, BNN_SCALE_E8M0, b_scale_ld, 1, K, S);
    if (st != BNN_OK) return st;
  }
  if (!offsets || !dw) return BNN_ERR_NULL;
  if (!aligned16(offsets) || !aligned16(dw)) return BNN_ERR_ALIGN;
  p.A = reinterpret_cast<const char *>(a), p.lda = lda, p.sa = a_scale, p.sa_ld = a_scale_ld;
  p.M = (int)N, p.N = (int)K, p.blocks = (int)f8_blocks(S), p.y = dw, p.type = type, p.ldy = dw_ld;
  p.groups = F8_GROUP_K, p.offsets = offsets, p.E = (int)experts, p.y_es = dw_expert_ld;
  return run_f8<false>(p, static_cast<hipStream_t>(stream));
}
