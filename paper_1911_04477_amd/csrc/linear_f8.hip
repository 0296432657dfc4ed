// Products of e4m3 matrices with block scales: the linear layer (bnn_linear_f8), the same for rows sorted by expert with a
// weight for each (bnn_expert_linear_f8), and the gradients of such weights (bnn_expert_linear_f8_dw).
#include <algorithm>

#include "bnn_testing.h"
#include "f8_mm.h"
#include "few_mm.h"

namespace bnn {

// Which kernel takes a product: that of few rows, or the tiles with the least time by what a round of them was measured to take, in us, with
// k of b blocks: start + block * b.  one: a compute unit has one tile at a time; two: it has two.  A last round of few tiles takes 0.55 of a round and
// more (f8_form; 8192 x 4096 to 2048, one round, 61 us, to 2304, a ninth more tiles, 95).  Over 84 sizes drawn at random the form taken is
// on average 3 % slower than the best of them.  Measured in bf16, scales powers of two, fast sums (exact ones in brackets), us:
//   rows x columns x k     256x256    256x128    128x128    the same, short k    128x128, one    128x64    64x64      64x32
//   64 x 4096 x 4096       37 (67)       24      23 (31)        22 (27)              17         12 (18)   10 (17)    8.5 (10)
//   256 x 4096 x 4096      41 (69)       27      24 (32)        23 (27)              18         14 (19)   11 (17)    16 (18)
//   512 x 4096 x 4096      41 (69)       27      24 (33)        23 (28)              18         14 (21)   16 (24)    29 (35)
//   1000 x 3001 x 2321     30 (48)       19      17 (23)        16 (20)              13.5       19 (25)   16 (23)    32 (38)
//   2048 x 4096 x 4096     42 (74)       34      34 (59)        34 (60)              39         52 (78)   54 (85)   110 (133)
//   8192 x 8192 x 2048    124 (205)     138     134 (226)      137 (233)            166        302 (368) 261 (368)
//   8192 x 4096 x 512      30 (41)       32      29 (39)        28 (39)              39         63 (76)   55 (65)
// 128 x 128 tiles come in three: two a unit of four waves each, two a unit of eight waves, whose starts and ends hide each other's better (short
// k), and one a unit with four steps in LDS.  256 x 256 tiles also come with their last round in quarters (launch_f8_rest).
enum : int { F8_256, F8_256_128, F8_128, F8_128_SHORT, F8_128_ONE, F8_128_64, F8_64, F8_64_32, F8_FORM_COUNT, F8_256_REST = F8_FORM_COUNT, F8_FEW };
struct F8Cost {
  float start, block, start2, block2;  // of one tile a unit, of two (0: one at a time)
};
struct F8Form {
  int bm, bn;
  F8Cost fast, exact, fast_wide, exact_wide;
};
constexpr F8Cost F8_NEVER = {1e9f, 0.0f, 0.0f, 0.0f};  // another is always faster
constexpr F8Form F8_FORMS[F8_FORM_COUNT] = {
    {256, 256, {12, 1.5f, 0, 0}, {19, 2.67f, 0, 0}, F8_NEVER, F8_NEVER},
    {256, 128, {5, 1.0f, 0, 0}, F8_NEVER, {6, 1.28f, 0, 0}, {9, 2.1f, 0, 0}},
    {128, 128, {3.5f, 0.73f, 4.5f, 1.07f}, {6, 0.86f, 8, 1.58f}, {3.5f, 0.85f, 4.5f, 1.65f}, F8_NEVER},
    {128, 128, {3.5f, 0.73f, 1.8f, 1.3f}, {5, 0.78f, 8.2f, 1.6f}, {3.5f, 0.8f, 3.5f, 1.8f}, {5, 1.05f, 10.5f, 2.2f}},
    {128, 128, {3.5f, 0.58f, 0, 0}, F8_NEVER, F8_NEVER, F8_NEVER},
    {128, 64, {3, 0.37f, 0, 0}, {4, 0.6f, 0, 0}, {3.5f, 0.5f, 0, 0}, F8_NEVER},
    {64, 64, {2.5f, 0.3f, 2.5f, 0.5f}, {3, 0.4f, 3, 0.65f}, {2.5f, 0.4f, 2.5f, 0.6f}, {3, 0.5f, 3, 0.8f}},
    {64, 32, {2.2f, 0.2f, 0, 0}, {2.5f, 0.25f, 0, 0}, {2.5f, 0.25f, 0, 0}, {2.5f, 0.3f, 0, 0}}};
constexpr F8Cost F8_QUARTERS = {3.5f, 0.58f, 0, 0}, F8_QUARTERS_EXACT = {5, 0.82f, 0, 0};
// rows: of all groups, or where these are along k (`same`) of each; blocks: of k a group.
inline int f8_form(int64_t rows, int64_t groups, bool same, int64_t N, int64_t blocks, bool wide, bool exact, int64_t units) {
  // Few rows: sixteen of A cost what sixteen of B do, so more than a few want tiles where there is enough to stream (16 rows of two
  // experts, 8192 x 4096 each: 17 us, on 64 x 64 tiles with fast sums 13), and fewer columns than units can keep busy want k split (one row, 4096 x
  // 4096: 6.0, 11).  Exact sums cost tiles more, fp32 scales on top of them more still, so that up to 8 and 12 rows stay here where the weights are
  // long (exact, few rows and 64 x 64 tiles: 8 rows, 16384 x 4096, 15.4 and 17.2 us, with fp32 scales 12 rows 17 and 26); below 16 MB either takes as
  // long, give or take a microsecond or two.  Rows of experts are uneven, and an expert's weights are read once for 16 rows: 128 rows of 16 experts,
  // 4096 x 4096, take 59 and 73 evenly spread, 60 and 50 where every expert has a quarter of what the one of half its rank has, so 8 rows on
  // average stay with fp32 scales only (64 rows of 8 experts, 33 and 42).
  const int64_t each = same ? rows : (rows - 1) / groups + 1, columns = groups * ((N - 1) / 16 + 1);
  const bool uneven = groups > 1 && !same, streamed = groups * N * blocks >= (16 << 20) / F8_BLOCK;
  const int64_t few = !exact || !streamed ? 4 : uneven ? (wide ? 8 : 4) : wide ? 12 : 8;
  if (each <= few || (each <= 16 && columns <= 2 * units)) return F8_FEW;
  int best = F8_64;
  double least = 1e30;
  for (int f = 0; f < F8_FORM_COUNT; ++f) {
    const F8Form &t = F8_FORMS[f];
    const F8Cost &c = wide ? (exact ? t.exact_wide : t.fast_wide) : exact ? t.exact : t.fast;
    int64_t row_tiles = groups * ((rows - 1) / t.bm + 1);
    if (groups > 1 && !same) row_tiles = std::max(groups * ((rows - 1) / (groups * t.bm) + 1), rows / t.bm + groups / 2);  // groups end inside tiles
    const int64_t tiles = row_tiles * ((N - 1) / t.bn + 1), rounds = tiles / units, rest = tiles % units;
    const auto in_rounds = [&](int64_t slots) {  // a last round that is not full has units, or the ways to them, to itself
      const double r = (double)(tiles % slots) / slots;
      return tiles <= slots ? 1.0 : tiles / slots + (r > 0 ? 0.55 + 0.45 * r : 0.0);
    };
    const double round = c.start + c.block * blocks, one = in_rounds(units) * round;
    const double two = tiles > units && c.block2 > 0 ? in_rounds(2 * units) * (c.start2 + c.block2 * blocks) : 1e30;
    if (std::min(one, two) < least) least = std::min(one, two), best = f;
    if (f == F8_256 && !wide && tiles > units) {
      const bool quarters = rest && rest * 4 <= units;  // as f8_whole
      const F8Cost &q = exact ? F8_QUARTERS_EXACT : F8_QUARTERS;
      const double time = quarters ? rounds * round + q.start + q.block * blocks + 2.0 : one;
      // How many tiles uneven groups fill is found on the device; where the second launch has nothing to do, it costs 2 us.
      if (time < one || (groups > 1 && !same)) least = std::min(time, one), best = F8_256_REST;
    }
  }
  return best;
}

template <int BM, int BN, int WGM, int WGN, int KG, int STAGES, bool WIDE, class E, bool EXACT>
bnn_status launch_f8_tile(F8Operands p, hipStream_t s) {
  p.tilesN = (p.N - 1) / BN + 1;
  // groups of rows: each has a part of a tile more than its rows fill at most
  p.tilesM = p.groups == F8_GROUP_ROWS ? p.M / BM + std::min(p.E, p.M) : (p.M - 1) / BM + 1;
  const int64_t tiles = (int64_t)p.tilesM * p.tilesN * (p.groups == F8_GROUP_K ? p.E : 1);
  if ((int64_t)p.tilesM * p.tilesN > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  ProfScope ps(KID_LINEAR_F8, s);
  wide_launches(tiles, [&](int64_t first, uint32_t n) {
    p.first = first;
    f8_tile_kernel<BM, BN, WGM, WGN, KG, STAGES, WIDE, E, EXACT><<<n, 64 * WGM * WGN * KG, 0, s>>>(p);
  });
  return launch_status();
}

// 256 x 256 tiles as far as they fill rounds of the units, and where few are left for a last one, quarters of those in a launch behind: these take
// a third of its time (fast sums: 8192 x 4096 to 2304 95 us as 256 x 256, 87 as 128 x 128, 76 so; 8192 rows of eight experts of uneven parts to
// 2048 108, 106, 92; exact 163, 134, 126).  How many there are of groups of rows, the kernels find for themselves.
template <class E, bool EXACT>
bnn_status launch_f8_rest(F8Operands p, hipStream_t s) {
  p.units = device_cu_count();
  const bnn_status st = launch_f8_tile<256, 256, 2, 2, 1, 2, false, E, EXACT>(p, s);
  if (st != BNN_OK) return st;
  p.tilesN = (p.N - 1) / 256 + 1;
  p.tilesM = p.groups == F8_GROUP_ROWS ? p.M / 256 + std::min(p.E, p.M) : (p.M - 1) / 256 + 1;
  p.first = 0;
  ProfScope ps(KID_LINEAR_F8, s);
  f8_tile_kernel<128, 128, 4, 2, 1, 4, false, E, EXACT, true><<<(p.units / 4 + 7) / 8 * 32, 512, 0, s>>>(p);
  return launch_status();
}

template <int SPLIT, bool WIDE>
bnn_status launch_f8_few_split(F8Operands p, int64_t row_tiles, hipStream_t s) {
  p.tilesN = (p.N - 1) / (128 / SPLIT) + 1;
  p.tilesM = (int)row_tiles;
  if (row_tiles * p.tilesN > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  ProfScope ps(KID_LINEAR_F8_FEW, s);
  wide_launches(row_tiles * p.tilesN * (p.groups == F8_GROUP_K ? p.E : 1), [&](int64_t first, uint32_t n) {
    p.first = first;
    f8_few_kernel<SPLIT, WIDE><<<n, 512, 0, s>>>(p);
  });
  return launch_status();
}
template <bool WIDE>
bnn_status launch_f8_few(const F8Operands &p, hipStream_t s) {
  const int64_t row_tiles = p.groups == F8_GROUP_ROWS ? p.M / 16 + std::min(p.E, p.M) : (p.M - 1) / 16 + 1;
  const int64_t columns = (row_tiles * (p.groups == F8_GROUP_K ? p.E : 1) * ((p.N - 1) / 16 + 1)), units = device_cu_count();
  if (columns >= 4 * units) return launch_f8_few_split<2, WIDE>(p, row_tiles, s);
  if (columns >= 2 * units) return launch_f8_few_split<4, WIDE>(p, row_tiles, s);
  return launch_f8_few_split<8, WIDE>(p, row_tiles, s);
}

template <bool WIDE, class E, bool EXACT>
bnn_status run_f8_as(const F8Operands &p, hipStream_t s) {
  const bool along_k = p.groups == F8_GROUP_K;
  const int64_t groups = p.groups == F8_PLAIN ? 1 : along_k ? p.E : std::min(p.E, p.M);
  switch (f8_form(p.M, groups, along_k, p.N, along_k ? p.blocks / p.E + 1 : p.blocks, WIDE, EXACT, device_cu_count())) {
    case F8_256:
      if constexpr (!WIDE) return launch_f8_tile<256, 256, 2, 2, 1, 2, false, E, EXACT>(p, s);
      break;
    case F8_256_REST:
      if constexpr (!WIDE) return launch_f8_rest<E, EXACT>(p, s);
      break;
    case F8_256_128:
      if constexpr (WIDE || !EXACT) return launch_f8_tile<256, 128, 4, 2, 1, 3, WIDE, E, EXACT>(p, s);
      break;
    case F8_128:
      if constexpr (!WIDE || !EXACT) return launch_f8_tile<128, 128, 2, 2, 1, 2, WIDE, E, EXACT>(p, s);
      break;
    case F8_128_SHORT: return launch_f8_tile<128, 128, 2, 4, 1, 2, WIDE, E, EXACT>(p, s);
    case F8_128_ONE:
      if constexpr (!WIDE && !EXACT) return launch_f8_tile<128, 128, 4, 2, 1, 4, false, E, EXACT>(p, s);
      break;
    case F8_128_64:
      if constexpr (!WIDE || !EXACT) return launch_f8_tile<128, 64, 2, 2, 2, 3, WIDE, E, EXACT>(p, s);
      break;
    case F8_64: return launch_f8_tile<64, 64, 2, 2, 1, 4, WIDE, E, EXACT>(p, s);
    case F8_64_32: return launch_f8_tile<64, 32, 2, 1, 4, 3, WIDE, E, EXACT>(p, s);
    default: return launch_f8_few<WIDE>(p, s);
  }
  return BNN_ERR_UNSUPPORTED;  // not reached: these forms are never the fastest (F8_NEVER)
}
template <bool WIDE>
bnn_status run_f8(const F8Operands &p, hipStream_t s) {
  if (p.fast) return run_f8_as<WIDE, __bf16, false>(p, s);
  return with_float(p.type, [&](auto tag) { return run_f8_as<WIDE, typename decltype(tag)::type, true>(p, s); });
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

// The type of results without the choice of their sums.
bnn_status f8_type(F8Operands &p, int type) {
  p.fast = type == (BNN_BF16 | BNN_FAST_SUMS);
  p.type = p.fast ? BNN_BF16 : type;
  return float_type(p.type) ? BNN_OK : BNN_ERR_SHAPE;
}

}  // namespace bnn

extern "C" bnn_status bnn_linear_f8(const uint8_t *a, int64_t lda, const uint8_t *a_scale, int64_t a_scale_ld, const uint8_t *b,
                                    int64_t ldb, const void *b_scale, int b_scale_type, int64_t b_scale_ld, int b_scale_rows,
                                    const float *bias, int64_t M, int64_t N, int64_t K, void *y, int type, int64_t ldy,
                                    void *stream) {
  using namespace bnn;
  F8Operands p = {};
  if (M < 0 || N < 0 || K <= 0 || f8_type(p, type) != BNN_OK) return BNN_ERR_SHAPE;
  if (ldy < N) return BNN_ERR_STRIDE;
  if (M > F8_MOST || N > F8_MOST || K > F8_MOST_K) return BNN_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return BNN_OK;
  bnn_status st = f8_check(a, lda, a_scale, a_scale_ld, K);
  if (st == BNN_OK) st = f8_weight(p, b, ldb, b_scale, b_scale_type, b_scale_ld, b_scale_rows, N, K);
  if (st != BNN_OK) return st;
  if (!y) return BNN_ERR_NULL;
  if (!aligned16(y) || !aligned4(bias)) return BNN_ERR_ALIGN;
  p.A = reinterpret_cast<const char *>(a), p.lda = lda, p.sa = a_scale, p.sa_ld = a_scale_ld;
  p.M = (int)M, p.blocks = (int)f8_blocks(K), p.bias = bias, p.y = y, p.ldy = ldy;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return b_scale_type == BNN_SCALE_F32 ? run_f8<true>(p, s) : run_f8<false>(p, s);
}

extern "C" bnn_status bnn_expert_linear_f8(const uint8_t *a, int64_t lda, const uint8_t *a_scale, int64_t a_scale_ld,
                                           const int32_t *offsets, int64_t experts, const uint8_t *b, int64_t ldb, int64_t b_expert_ld,
                                           const void *b_scale, int b_scale_type, int64_t b_scale_ld, int64_t b_scale_expert_ld,
                                           int b_scale_rows, int64_t S, int64_t N, int64_t K, void *y, int type, int64_t ldy,
                                           void *stream) {
  using namespace bnn;
  F8Operands p = {};
  if (S < 0 || N < 0 || K <= 0 || experts < 0 || f8_type(p, type) != BNN_OK) return BNN_ERR_SHAPE;
  if (ldy < N) return BNN_ERR_STRIDE;
  if (S > F8_MOST || N > F8_MOST || K > F8_MOST_K || experts > 65535) return BNN_ERR_UNSUPPORTED;
  if (S == 0 || N == 0 || experts == 0) return BNN_OK;
  bnn_status st = f8_check(a, lda, a_scale, a_scale_ld, K);
  if (st == BNN_OK) st = f8_weight(p, b, ldb, b_scale, b_scale_type, b_scale_ld, b_scale_rows, N, K);
  if (st != BNN_OK) return st;
  const int64_t scale_rows = b_scale_rows == 1 ? N : f8_blocks(N);
  if (experts > 1 && (b_expert_ld / N < ldb || b_expert_ld % 16 || b_scale_expert_ld / scale_rows < b_scale_ld || (b_scale_type == BNN_SCALE_E8M0 && b_scale_expert_ld % 4)))
    return BNN_ERR_STRIDE;
  if (!offsets || !y) return BNN_ERR_NULL;
  if (!aligned4(offsets) || !aligned16(y)) return BNN_ERR_ALIGN;
  p.A = reinterpret_cast<const char *>(a), p.lda = lda, p.sa = a_scale, p.sa_ld = a_scale_ld;
  p.M = (int)S, p.blocks = (int)f8_blocks(K), p.y = y, p.ldy = ldy;
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
  F8Operands p = {};
  if (S < 0 || N < 0 || K < 0 || experts < 0 || f8_type(p, type) != BNN_OK) return BNN_ERR_SHAPE;
  if (dw_ld < K || (experts > 1 && N > 0 && dw_expert_ld / N < dw_ld)) return BNN_ERR_STRIDE;
  if (S > F8_MOST_K || N > F8_MOST || K > F8_MOST || experts > 65535) return BNN_ERR_UNSUPPORTED;
  if (N == 0 || K == 0 || experts == 0) return BNN_OK;
  if (S > 0) {  // else every group is empty, and the result 0
    bnn_status st = f8_check(a, lda, a_scale, a_scale_ld, S);
    if (st == BNN_OK) st = f8_weight(p, b, ldb, b_scale, BNN_SCALE_E8M0, b_scale_ld, 1, K, S);
    if (st != BNN_OK) return st;
  }
  if (!offsets || !dw) return BNN_ERR_NULL;
  if (!aligned4(offsets) || !aligned16(dw)) return BNN_ERR_ALIGN;
  p.A = reinterpret_cast<const char *>(a), p.lda = lda, p.sa = a_scale, p.sa_ld = a_scale_ld;
  p.M = (int)N, p.N = (int)K, p.blocks = (int)f8_blocks(S), p.y = dw, p.ldy = dw_ld;
  p.groups = F8_GROUP_K, p.offsets = offsets, p.E = (int)experts, p.y_es = dw_expert_ld;
  return run_f8<false>(p, static_cast<hipStream_t>(stream));
}

extern "C" int bnn_testing_f8_form(int64_t rows, int64_t groups, int along_k, int64_t N, int64_t K, int scale_type, int type, int units) {
  using namespace bnn;
  if (rows <= 0 || groups <= 0 || N <= 0 || K <= 0 || !float_type(type) || units <= 0) return -1;
  return f8_form(rows, groups, along_k != 0, N, f8_blocks(K), scale_type == BNN_SCALE_F32, type != BNN_BF16, units);
}
