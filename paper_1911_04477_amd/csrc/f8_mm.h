// Matrix-core product of two row-major operands in e4m3 with a scale for each block of 128 values (f8.h),
//   y[m][n] = sum over blocks of scaleA[m][b] * scaleB[n][b] * (sum over the block's k of A[m][k] * B[n][k]),
// fp32 sums.  A step of 128 bytes of k is one block.  Scales that are powers of two go into the matrix instruction as bytes, or into the widening;
// fp32 scales of B, one for 128 rows and a block, multiply a block's sums on the vector unit (the rows' scale is in them by then).  These
// multiply-adds, 16 for two matrix instructions (eight where sums are EXACT), come behind all products of a step and are not hidden by them, and a
// block's own sums take as many registers as the tile's, so that tiles are 256 x 128 at most: 8192^3 in bf16 1060 us for 715, with FAST sums 740 for 459.
//
// Sums are EXACT: values go to bf16 on their way into the 16-bit matrix instruction, times their scales; no digit is lost, and sums are fp32's.
//
// bf16 results may be asked for with FAST sums, up to twice as fast (8192^3 444 to 483 us, EXACT 715): the 8-bit matrix instruction is exact in single
// products and adds up groups of them in fp32, but of the products of eight consecutive k it keeps no bits below 2^-13 of the largest.  A
// result is off by less than 2^-10 of the sum of its products' magnitudes, for normal values by 1.5e-5 of itself in the 2-norm, whatever the length:
// a hundredth of what rounding it to bf16 costs, but more where terms cancel; and where a result is quantised again, values next to
// a border go to the other side of it (a layer of experts in bf16 is off by 0.0028 for 0.0017).  So it is the caller's choice (BNN_FAST_SUMS).  The
// kernel of few rows is bound by memory and always EXACT.
//
// The same kernels take the experts' products: rows of A in groups with a weight each, or groups along k with a result each.
#pragma once
#include "f8.h"
#include "tile_mm.h"

namespace bnn {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

enum F8Groups : int { F8_PLAIN = 0, F8_GROUP_ROWS = 1, F8_GROUP_K = 2 };

struct F8Operands {
  const char *A, *B;
  int64_t lda, ldb;  // bytes between rows
  const uint8_t *sa;
  const void *sb;    // bytes, or fp32
  int64_t sa_ld, sb_ld;
  int sb_shift;      // rows of B that share a row of scales: 2^sb_shift
  const float *bias;
  void *y;
  int64_t ldy;
  int type;
  bool fast;  // sums
  int M, N, blocks;
  int tilesM, tilesN;
  int64_t first;     // tile of this launch's first workgroup
  int units;         // compute units, where a last round of few tiles is left to a second launch (f8_whole); 0: it is not
  // groups
  int groups;        // F8Groups
  const int32_t *offsets;  // [E + 1]
  int E;
  int64_t b_es, sb_es, y_es;  // between experts: bytes, bytes, elements
};

// One group's part of a call, as a workgroup sees it.
struct F8Part {
  const char *A, *B;
  const uint8_t *sa, *sb;
  int readable;        // bytes of a row of scales
  int first;           // block of k
  char *y;
  int m0, n0, M, N;    // first row and column; the ends
  int blocks;
};

// Tiles of rows by group: those before each group from a scan over the experts' counts, 64 at a time.  A launch has workgroups for as
// many tiles as there can be; those beyond end.
struct F8Group {
  int e, lo, hi, tile;  // expert, its first row and its end, the tile among its own
};
__device__ __forceinline__ int f8_clamped(const int32_t *offsets, int e, int S) { return min(max(offsets[e], 0), S); }
struct F8Scan {
  int lo, hi, sum;  // of this lane's expert; tiles up to and with its own
  template <int BM>
  __device__ __forceinline__ void run(const F8Operands &p, int e0) {
    const int lane = threadIdx.x & 63, e = e0 + lane;
    lo = e < p.E ? f8_clamped(p.offsets, e, p.M) : 0;
    hi = e < p.E ? max(f8_clamped(p.offsets, e + 1, p.M), lo) : 0;
    sum = (hi - lo + BM - 1) / BM;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
  }
  __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(sum, 63); }
  __device__ __forceinline__ bool find(int wanted, int e0, F8Group &g) const {
    const uint64_t past = __ballot(sum > wanted);
    if (!past) return false;
    const int l = __builtin_ctzll(past);
    g = {e0 + l, __builtin_amdgcn_readlane(lo, l), __builtin_amdgcn_readlane(hi, l), wanted - (l ? __builtin_amdgcn_readlane(sum, l - 1) : 0)};
    return true;
  }
};
template <int BM>
__device__ __forceinline__ int f8_row_tiles(const F8Operands &p) {
  int all = 0;
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    F8Scan scan;
    scan.run<BM>(p, e0);
    all += scan.total();
  }
  return all;
}
template <int BM>
__device__ __forceinline__ bool f8_row_group(const F8Operands &p, int wanted, F8Group &g) {
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    F8Scan scan;
    scan.run<BM>(p, e0);
    if (scan.find(wanted, e0, g)) return true;
    wanted -= scan.total();
  }
  return false;
}

// Of `tiles`, those that this launch takes whole: all, or where what is left behind full rounds makes at most a round of quarters, the full rounds.
__host__ __device__ __forceinline__ int64_t f8_whole(int64_t tiles, int units) {
  if (units == 0) return tiles;
  const int64_t rest = tiles % units;
  return rest * 4 <= units ? tiles - rest : tiles;
}

// The tile of a workgroup; false: none is left for it.  BM x BN outputs.  STREAMED: B is read once, so tiles of a group follow each other.
// REST: ids count from the tiles on that the first launch did not take.
template <int BM, int BN, bool STREAMED = false, bool REST = false>
__device__ __forceinline__ bool f8_part(const F8Operands &p, int64_t id, F8Part &t) {
  const auto taken = [&](int64_t tiles) {
    const int64_t whole = f8_whole(tiles, p.units);
    if (REST) id += whole;
    return id < (REST ? tiles : whole);
  };
  int tm, tn;
  const int size = p.type == BNN_F32 ? 4 : 2, readable = (p.blocks + 3) & ~3;
  if (p.groups == F8_GROUP_ROWS) {
    F8Group g;
    if (STREAMED) {
      tm = (int)(id / p.tilesN), tn = (int)(id - (int64_t)tm * p.tilesN);
      if (!f8_row_group<BM>(p, tm, g)) return false;
    } else if (p.E <= 64) {
      F8Scan scan;
      scan.run<BM>(p, 0);
      const int tilesM = scan.total();
      if (!taken((int64_t)tilesM * p.tilesN)) return false;
      mm_tile((int)id, tilesM, p.tilesN, tm, tn);
      scan.find(tm, 0, g);
    } else {
      const int tilesM = f8_row_tiles<BM>(p);
      if (!taken((int64_t)tilesM * p.tilesN)) return false;
      mm_tile((int)id, tilesM, p.tilesN, tm, tn);
      f8_row_group<BM>(p, tm, g);
    }
    t = {p.A, p.B + g.e * p.b_es, p.sa, static_cast<const uint8_t *>(p.sb) + g.e * p.sb_es, readable, 0, static_cast<char *>(p.y),
         g.lo + g.tile * BM, tn * BN, g.hi, p.N, p.blocks};
    return true;
  }
  const int64_t of = (int64_t)p.tilesM * p.tilesN;
  if (p.groups == F8_GROUP_K) {
    if (!taken(of * p.E)) return false;
    const int e = (int)(id / of);
    mm_tile((int)(id - e * of), p.tilesM, p.tilesN, tm, tn);
    const int end = p.blocks * F8_BLOCK, lo = f8_clamped(p.offsets, e, end) / F8_BLOCK, hi = max(f8_clamped(p.offsets, e + 1, end) / F8_BLOCK, lo);
    t = {p.A + (int64_t)lo * F8_BLOCK, p.B + (int64_t)lo * F8_BLOCK, p.sa, static_cast<const uint8_t *>(p.sb), readable, lo,
         static_cast<char *>(p.y) + e * p.y_es * size, tm * BM, tn * BN, p.M, p.N, hi - lo};
    return true;
  }
  if (!taken(of)) return false;
  mm_tile((int)id, p.tilesM, p.tilesN, tm, tn);
  t = {p.A, p.B, p.sa, static_cast<const uint8_t *>(p.sb), readable, 0, static_cast<char *>(p.y), tm * BM, tn * BN, p.M, p.N, p.blocks};
  return true;
}

// The scales of four blocks of a row from block kb on; past the row's bytes nothing is read.
__device__ __forceinline__ uint32_t f8_scales(const uint8_t *row, int kb, int end) {
  typedef uint32_t u32_any __attribute__((aligned(1)));
  const int at = min(kb, end - 4);
  return *reinterpret_cast<const u32_any *>(row + at) >> (8 * (kb - at));
}

// Four e4m3 values times 2^p as bf16, both exactly.
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void f8_widen(int four, float scale, v8bf &to, int at) {
  const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true);
  to[at] = lo[0], to[at + 1] = lo[1], to[at + 2] = hi[0], to[at + 3] = hi[1];
}
struct F8Wide {
  v8bf v[4];
  __device__ __forceinline__ void set(const v8i &q, uint32_t scale) {  // scale: p + 127
    const float s = __uint_as_float(scale << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) f8_widen(q[i], s, v[i / 2], i % 2 * 4);
  }
};

__device__ __forceinline__ v16f f8_mfma(const v8i &a, const v8i &b, const v16f &c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}

// A wave's 16 accumulators of a 256 x 256 tile fill the accumulation registers (mm_settle in tile_mm.h): products written out, each in place.
__device__ __forceinline__ void f8_mfma_in_place(const v8i &a, const v8i &b, v16f &c, uint32_t sa, uint32_t sb) {
  asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}
__device__ __forceinline__ void f8_settle(v16f (&c)[4]) {  // a matrix instruction of 16 passes: 19 wait states
  asm volatile("s_nop 15\n\ts_nop 7" : "+a"(c[0]), "+a"(c[1]), "+a"(c[2]), "+a"(c[3]));
}

// Reads of LDS, requests and what the vector unit does between MATRIX matrix instructions, not all in front of them.
template <int Q, int MATRIX, int READS, int LOADS, bool WIDENS>
__device__ __forceinline__ void f8_interleave() {
  if constexpr (Q == MATRIX) {
    __builtin_amdgcn_sched_barrier(0);
  } else {
    constexpr int R = READS * (Q + 1) / MATRIX - READS * Q / MATRIX, N = LOADS * (Q + 1) / MATRIX - LOADS * Q / MATRIX;
    if constexpr (WIDENS) __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
    if constexpr (R > 0) __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
    if constexpr (N > 0) __builtin_amdgcn_sched_group_barrier(0x010, N, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    f8_interleave<Q + 1, MATRIX, READS, LOADS, WIDENS>();
  }
}

// LDS: a step's rows of 128 bytes, 16-byte piece c of row r in slot c ^ (r / 2 % 8), so that the 16 rows of a clock spread over
// all 64 banks (with r % 8 a read takes twice as long); behind them for each row the
// four bytes of scales that hold the step's.  WGM x WGN waves of 32 x 32 blocks; KG such groups of waves take the blocks of k in turn, KG
// of them a step, and their sums meet in the end: small tiles, one a compute unit, are bound by what a step does one after the other
// (64 x 4096 by 4096 on 64 x 32 tiles, FAST, 9.9 us with one group, 8.6 with four).
template <int BM, int BN, int WGM, int WGN, int KG, int STAGES, bool WIDE>
struct F8Tile {
  static constexpr int WAVES = WGM * WGN, ROWS = BM + BN, SCALED = WIDE ? BM : ROWS, LOADS_A = BM / 8 / WAVES, LOADS_ROWS = ROWS / 8 / WAVES,
                       LOADS_SCALES = (SCALED / 64 + WAVES - 1) / WAVES, LOADS = LOADS_ROWS + (LOADS_SCALES ? LOADS_SCALES : 1),
                       PART = ROWS * MM_STEP + (SCALED + 63) / 64 * 256, STAGE = KG * PART, TM = BM / WGM / 32, TN = BN / WGN / 32;
  static_assert(ROWS % (8 * WAVES) == 0 && BM % (8 * WAVES) == 0 && BM % (32 * WGM) == 0 && BN % (32 * WGN) == 0, "");
};
// WIDE: fp32 scales of B; E: the results' type; EXACT: see above; QUARTERS: of the tiles of twice the size both ways that are left.
template <int BM, int BN, int WGM, int WGN, int KG, int STAGES, bool WIDE, class E, bool EXACT, bool QUARTERS>
__device__ __forceinline__ void f8_tile_product(const F8Operands &p, char *const whole_lds) {
  using L = F8Tile<BM, BN, WGM, WGN, KG, STAGES, WIDE>;
  constexpr int WAVES = L::WAVES, LOADS = L::LOADS, STAGE = L::STAGE, TM = L::TM, TN = L::TN;
  constexpr bool IN_PLACE = TM * TN == 16;
  F8Part t;
  if constexpr (QUARTERS) {  // the four of a tile on one XCD
    const int64_t id = p.first + blockIdx.x;
    if (!f8_part<2 * BM, 2 * BN, false, true>(p, (id >> 5) * 8 + (id & 7), t)) return;
    t.m0 += (int)(id >> 4 & 1) * BM, t.n0 += (int)(id >> 3 & 1) * BN;
    if (t.m0 >= t.M || t.n0 >= t.N) return;
  } else {
    if (!f8_part<BM, BN>(p, p.first + blockIdx.x, t)) return;
  }
  const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = id / WAVES, wave = id % WAVES;
  const int wm = wave / WGN, wn = wave % WGN;
  char *const lds = whole_lds + group * L::PART;
  const auto piece = [&](int load) { return ((lane & 7) ^ (lane >> 4) ^ (load & 1) * 4) * 16; };  // of a step's 128 bytes, that this lane brings
  const auto resA = __builtin_amdgcn_make_buffer_rsrc((void *)(t.A + (int64_t)t.m0 * p.lda), 0, 0xffffffffu, 0x00020000);
  const auto resB = __builtin_amdgcn_make_buffer_rsrc((void *)(t.B + (int64_t)t.n0 * p.ldb), 0, 0xffffffffu, 0x00020000);
  const auto resSA = __builtin_amdgcn_make_buffer_rsrc((void *)(t.sa + (int64_t)t.m0 * p.sa_ld), 0, 0xffffffffu, 0x00020000);
  const auto resSB = __builtin_amdgcn_make_buffer_rsrc((void *)(t.sb + (WIDE ? 0 : (int64_t)(t.n0 >> p.sb_shift) * p.sb_ld)), 0, 0xffffffffu, 0x00020000);
  uint32_t at[LOADS];  // rows beyond the operands repeat the last one, their outputs are not stored
  const auto is_scale = [](int i) { return i >= L::LOADS_ROWS; };
  const auto scale_row = [&](int i) { return min((i - L::LOADS_ROWS) * WAVES + wave, (L::SCALED + 63) / 64 - 1) * 64; };  // first of a load
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    if (!is_scale(i)) {
      const int load = i * WAVES + wave, row = load * 8 + (lane >> 3);
      at[i] = i < L::LOADS_A ? __umul24(min(row, t.M - 1 - t.m0), (uint32_t)p.lda) + piece(load)  // strides are below 2^22
                             : __umul24(min(row - BM, t.N - 1 - t.n0), (uint32_t)p.ldb) + piece(load);
    } else {
      const int row = min(scale_row(i) + lane, L::SCALED - 1);
      at[i] = row < BM ? __umul24(min(row, t.M - 1 - t.m0), (uint32_t)p.sa_ld)
                       : __umul24((min(t.n0 + row - BM, t.N - 1) >> p.sb_shift) - (t.n0 >> p.sb_shift), (uint32_t)p.sb_ld);
    }
  }
  static_assert(BM % 64 == 0, "a load of scales is of one operand");
  const auto request_one = [&](int i, int step, char *lds) {
    using To = __attribute__((address_space(3))) void *;
    if (is_scale(i)) {
      const int row = scale_row(i), k = (t.first + step) & ~3;
      const To to = (To)(lds + L::ROWS * MM_STEP + row * 4);
      if (row < BM) __builtin_amdgcn_raw_ptr_buffer_load_lds(resSA, to, 4, at[i], k, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(resSB, to, 4, at[i], k, 0, 0);
    } else {
      const To to = (To)(lds + (i * WAVES + wave) * 8 * MM_STEP);
      if (i < L::LOADS_A) __builtin_amdgcn_raw_ptr_buffer_load_lds(resA, to, 16, at[i], step * MM_STEP, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(resB, to, 16, at[i], step * MM_STEP, 0, 0);
    }
  };
  const auto block_of = [&](int step) { return KG == 1 ? step : min(step * KG + group, t.blocks - 1); };  // past the end: not used
  const auto request = [&](int step, char *lds) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) request_one(i, block_of(step), lds);
  };
  const int steps = (t.blocks + KG - 1) / KG;
  for (int i = 0; i < min(steps, STAGES); ++i) request(i, lds + i * STAGE);

  const float *wide[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) {  // the first of 32 columns, which share an fp32 scale
    const int n = min(t.n0 + wn * (BN / WGN) + j * 32, t.N - 1);
    wide[j] = WIDE ? reinterpret_cast<const float *>(t.sb) + (int64_t)__builtin_amdgcn_readfirstlane(n >> 7) * p.sb_ld : nullptr;
  }
  v16f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v16f{};
  if (p.bias && group == 0) {  // sums start from it
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float v = p.bias[min(t.n0 + wn * (BN / WGN) + j * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, t.N - 1)];
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j][r] = v;
      }
  }
  if constexpr (IN_PLACE && !EXACT)
#pragma unroll
    for (int i = 0; i < TM; ++i) f8_settle(acc[i]);
  // Lanes 0 to 31 have pieces 0, 1 of a half step's four, the others 2, 3.
  const int slot = (((lane >> 5) * 2) ^ (lane >> 1 & 7)) * 16;
  const int rowA = wm * (BM / WGM) + (lane & 31), rowB = BM + wn * (BN / WGN) + (lane & 31);
  const int fragA = rowA * MM_STEP + slot, fragB = rowB * MM_STEP + slot;
  struct Half {  // fragments of 64 bytes of k
    v4i a[TM][2], b[TN][2];
  };
  struct Scales {
    uint32_t a[TM], b[TN];
  };
  // The k-th read of a half step: B's pieces, A's, then with the first half the step's scales.
  constexpr int PIECES = 2 * (TM + TN), READS = PIECES + TM + (WIDE ? 0 : TN);
  const auto fetch_one = [&](Half &f, Scales &s, const char *lds, int block, int half, int k) {
    if (k < 2 * TN) f.b[k / 2][k % 2] = *reinterpret_cast<const v4i *>(lds + (fragB ^ (half * 64 + k % 2 * 16)) + k / 2 * 32 * MM_STEP);
    else if (k < PIECES) f.a[k / 2 - TN][k % 2] = *reinterpret_cast<const v4i *>(lds + (fragA ^ (half * 64 + k % 2 * 16)) + (k / 2 - TN) * 32 * MM_STEP);
    else {
      const uint8_t *scales = reinterpret_cast<const uint8_t *>(lds + L::ROWS * MM_STEP) + ((t.first + block) & 3);
      if (k < PIECES + TM) s.a[k - PIECES] = scales[(rowA + (k - PIECES) * 32) * 4];
      else s.b[k - PIECES - TM] = scales[(rowB + (k - PIECES - TM) * 32) * 4];
    }
  };
  const auto fetch = [&](Half &f, Scales &s, const char *lds, int step, int half) {
#pragma unroll
    for (int k = 0; k < (half ? PIECES : READS); ++k) fetch_one(f, s, lds, block_of(step), half, k);
  };
  const auto whole = [](const v4i (&v)[2]) { return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7); };
  v16f part[TM][TN];  // WIDE: a block's sums
  const auto multiply = [&](const Half &f, const Scales &s, int half) {
    if constexpr (EXACT) {
      const auto start = [&](int i, int j) { return !WIDE ? acc[i][j] : half ? part[i][j] : v16f{}; };
      F8Wide b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j].set(whole(f.b[j]), WIDE ? 127u : s.b[j]);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        F8Wide a;
        a.set(whole(f.a[i]), s.a[i]);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          v16f sum = start(i, j);
#pragma unroll
          for (int c = 0; c < 4; ++c) sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j].v[c], a.v[c], sum, 0, 0, 0);
          (WIDE ? part : acc)[i][j] = sum;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {  // rows of the result: n
          if constexpr (WIDE) part[i][j] = f8_mfma(whole(f.b[j]), whole(f.a[i]), half ? part[i][j] : v16f{}, 127u, s.a[i]);
          else acc[i][j] = f8_mfma(whole(f.b[j]), whole(f.a[i]), acc[i][j], s.b[j], s.a[i]);
        }
    }
  };
  const auto scale_parts = [&](int step) {
    if constexpr (WIDE)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const float w = wide[j][block_of(step)];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = fmaf(part[i][j][r], w, acc[i][j][r]);
      }
  };

  const auto interleave = [&](auto reads, auto loads) {
    constexpr int MATRIX = TM * TN * (EXACT ? 4 : 1);
    if constexpr (MATRIX >= 16) f8_interleave<0, MATRIX, decltype(reads)::value, decltype(loads)::value, EXACT>();
  };
  // As in tile_mm.h: the workgroup meets in the middle of a step, when both halves of its fragments are in registers; from there on
  // its place in LDS takes the step STAGES ahead, and the next step's first half is read under the products of the second.
  if (steps) {
    Half first, second;
    Scales scales[2];
    if (steps >= STAGES) mm_sync<(STAGES - 1) * LOADS>();
    else mm_sync<0>();
    fetch(first, scales[0], lds, 0, 0);
    int now = 0;
    // EXACT, 256 x 256: eight bytes of every fragment at a time are widened for 16 products, two instructions behind each product of
    // the 16 before.
    constexpr bool WOVEN = EXACT && IN_PLACE;
    struct Chunk {
      v8bf a[TM], b[TN];
    };
    Chunk chunk[2];
    float factors[2][TM + TN];
    const auto factor = [&](const Scales &s, float (&to)[TM + TN]) {
#pragma unroll
      for (int i = 0; i < TM; ++i) to[i] = __uint_as_float(s.a[i] << 23);
#pragma unroll
      for (int j = 0; j < TN; ++j) to[TM + j] = __uint_as_float(s.b[j] << 23);
    };
    const auto widen = [&](Chunk &to, const Half &f, const float (&by)[TM + TN], int c, int u) {  // the u-th of 2 * (TM + TN) parts; B first
      const int k = u / 2, w = c % 2 * 2 + u % 2;
      if (k < TN) f8_widen(f.b[k][c / 2][w], by[TM + k], to.b[k], u % 2 * 4);
      else f8_widen(f.a[k - TN][c / 2][w], by[k - TN], to.a[k - TN], u % 2 * 4);
    };
    if constexpr (WOVEN) {
      factor(scales[0], factors[0]);
#pragma unroll
      for (int u = 0; u < 16; ++u) widen(chunk[0], first, factors[0], 0, u);
    }
    const auto turn = [&](int i, Scales &mine, Scales &other, auto inside) {  // inside: known to be neither last nor among the last STAGES
      const int next = now + 1 == STAGES ? 0 : now + 1;
      const bool more = decltype(inside)::value || i + STAGES < steps, last = !decltype(inside)::value && i + 1 == steps;
      if constexpr (IN_PLACE && !EXACT) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          fetch_one(second, mine, lds + now * STAGE, i, 1, q);
          f8_mfma_in_place(whole(first.b[q % 4]), whole(first.a[q / 4]), acc[q / 4][q % 4], mine.b[q % 4], mine.a[q / 4]);
        }
        if (decltype(inside)::value || i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
        else mm_sync<0>();
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          if (!last) {
            fetch_one(first, other, lds + next * STAGE, i + 1, 0, q);
            if (q % 2 == 0) fetch_one(first, other, lds + next * STAGE, i + 1, 0, 16 + q / 2);
          }
          f8_mfma_in_place(whole(second.b[q % 4]), whole(second.a[q / 4]), acc[q / 4][q % 4], mine.b[q % 4], mine.a[q / 4]);
          if (more) {
            request_one(q, i + STAGES, lds + now * STAGE);
            if (q < LOADS - 16) request_one(16 + q, i + STAGES, lds + now * STAGE);
          }
        }
      } else if constexpr (WOVEN) {
        const int which = &mine == &scales[0] ? 0 : 1;
        const auto phase = [&](const Half &of, const Half &then, const float (&by)[TM + TN], const float (&then_by)[TM + TN], const auto &between) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              between(c * 16 + q);
              widen(chunk[(c + 1) % 2], c < 3 ? of : then, c < 3 ? by : then_by, (c + 1) % 4, q);
              acc[q / 4][q % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(chunk[c % 2].b[q % 4], chunk[c % 2].a[q / 4], acc[q / 4][q % 4], 0, 0, 0);
              __builtin_amdgcn_sched_barrier(0);
            }
        };
        phase(first, second, factors[which], factors[which], [&](int q) {
          if (q % 2 == 0 && q / 2 < PIECES) fetch_one(second, mine, lds + now * STAGE, i, 1, q / 2);
        });
        if (decltype(inside)::value || i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
        else mm_sync<0>();
        phase(second, first, factors[which], factors[which ^ 1], [&](int q) {
          if (q % 2 == 0 && q / 2 < READS && !last) fetch_one(first, other, lds + next * STAGE, i + 1, 0, q / 2);
          if (q % 2 == 1 && q / 2 < LOADS && more) request_one(q / 2, i + STAGES, lds + now * STAGE);
          if (q == 48) factor(other, factors[which ^ 1]);
        });
      } else {
        __builtin_amdgcn_sched_barrier(0);
        const bool any = decltype(inside)::value || i * KG + group < t.blocks;  // a block for this group
        fetch(second, mine, lds + now * STAGE, i, 1);
        if (any) multiply(first, mine, 0);
        if constexpr (decltype(inside)::value) interleave(std::integral_constant<int, PIECES>(), std::integral_constant<int, 0>());
        if (decltype(inside)::value || i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
        else mm_sync<0>();
        __builtin_amdgcn_sched_barrier(0);
        if (more) request(i + STAGES, lds + now * STAGE);
        if (!last) fetch(first, other, lds + next * STAGE, i + 1, 0);
        if (any) {
          multiply(second, mine, 1);
          if constexpr (decltype(inside)::value) interleave(std::integral_constant<int, READS>(), std::integral_constant<int, LOADS>());
          scale_parts(i);
        }
      }
      now = next;
    };
    int i = 0;
    for (; i + 1 + STAGES < steps; i += 2) {
      turn(i, scales[0], scales[1], std::true_type());
      turn(i + 1, scales[1], scales[0], std::true_type());
    }
    for (; i < steps; i += 2) {
      turn(i, scales[0], scales[1], std::false_type());
      if (i + 1 < steps) turn(i + 1, scales[1], scales[0], std::false_type());
    }
  }
  if constexpr (IN_PLACE && !EXACT)
#pragma unroll
    for (int i = 0; i < TM; ++i) f8_settle(acc[i]);

  if constexpr (KG > 1) {  // the groups' sums, in their order
    constexpr int SUMS = TM * TN * 16 * 64;  // a wave's
    static_assert((KG - 1) * WAVES * SUMS * 4 <= STAGES * STAGE, "");
    float *const sums = reinterpret_cast<float *>(whole_lds) + wave * (KG - 1) * SUMS + lane * 4;
    mm_meet();
    if (group) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<v4f *>(sums + (group - 1) * SUMS + ((i * TN + j) * 4 + q) * 256) =
                v4f{acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
    }
    mm_meet();
    if (group) return;
#pragma unroll
    for (int g = 1; g < KG; ++g)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const v4f v = *reinterpret_cast<const v4f *>(sums + (g - 1) * SUMS + ((i * TN + j) * 4 + q) * 256);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][q * 4 + r] += v[r];
          }
  }

  // Results leave through LDS, 32 rows of a wave's columns at a time, so that a store covers whole lines of a row.
  if constexpr (KG == 1) mm_meet();
  else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // a wave's own part of what it has just read
  constexpr int SIZE = sizeof(E), PITCH = TN * 32 * SIZE + 16, PARTS = TN * 32 * SIZE / 16, PER = 16 / SIZE;
  static_assert(WAVES * 32 * PITCH <= STAGES * STAGE && (KG == 1 || 32 * PITCH <= (KG - 1) * TM * TN * 16 * 64 * 4), "");
  char *const mine = KG == 1 ? lds + wave * 32 * PITCH : whole_lds + wave * (KG - 1) * (TM * TN * 16 * 64 * 4);  // where only this wave reads
  const int n0 = t.n0 + wn * (BN / WGN);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m0 = t.m0 + wm * (BM / WGM) + i * 32;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        // A lane has column m = lane % 32 of a block and four times four consecutive n, those of the lane 32 above in between: these
        // trade, so that a lane has eight consecutive ones.
        const int n = j * 32 + q * 8 + (lane >> 5) * 8;
        float v[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][q * 4 + r]), __float_as_uint(acc[i][j][q * 4 + 4 + r]), false, false);
          v[r] = __uint_as_float(two[0]), v[4 + r] = __uint_as_float(two[1]);
        }
        store8(reinterpret_cast<E *>(mine + (lane & 31) * PITCH), n, TN * 32, v);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int k = 0; k < PARTS / 2; ++k) {
      const int at = k * 64 + lane, row = at / PARTS, n = n0 + at % PARTS * PER, m = m0 + row;
      const char *from = mine + row * PITCH + at % PARTS * 16;
      const u32x4 v = *reinterpret_cast<const u32x4 *>(from);
      if (m >= t.M || n >= t.N) continue;
      E *to = reinterpret_cast<E *>(t.y) + m * p.ldy + n;
      if (n + PER <= t.N) {  // results of large tiles past the caches (8192 x 4096 to 4096, FAST, 122 -> 119 us)
        if constexpr (BM * BN >= 128 * 128) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any *>(to));
        else *reinterpret_cast<u32x4_any *>(to) = v;
      } else
        for (int r = 0; r < t.N - n; ++r) to[r] = reinterpret_cast<const E *>(from)[r];
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

template <int BM, int BN, int WGM, int WGN, int KG, int STAGES, bool WIDE, class E, bool EXACT, bool QUARTERS = false>
__global__ __launch_bounds__(64 * WGM *WGN *KG, WGM *WGN *KG < 4 ? 1 : WGM *WGN *KG / 4) void f8_tile_kernel(F8Operands p) {
  __shared__ __attribute__((aligned(16))) char lds[STAGES * F8Tile<BM, BN, WGM, WGN, KG, STAGES, WIDE>::STAGE];
  f8_tile_product<BM, BN, WGM, WGN, KG, STAGES, WIDE, E, EXACT, QUARTERS>(p, lds);
}

// At most 16 rows of A (of a group): nothing is reused, B is streamed once and bounds the kernel.  A wave owns 16 columns and deals with
// every SPLIT-th run of two blocks of k, straight from memory into registers, the next run requested before the products of the present one; the
// SPLIT waves of a column's sums meet in LDS.  Short-lived workgroups wait for their first loads most of their time, so k is split no
// further than it takes to give every unit waves (32 rows of eight experts, 8192 x 4096 each: split eight ways 73 us, two ways 57, 4.7 TB/s).
template <int SPLIT, bool WIDE>
__device__ __forceinline__ void f8_few_product(const F8Operands &p, v4f (*sums)[64]) {
  constexpr int WAVES = 8, COLUMNS = WAVES / SPLIT * 16;
  F8Part t;
  if (!f8_part<16, COLUMNS, true>(p, p.first + blockIdx.x, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = t.n0 + wave / SPLIT * 16, row = lane & 15, piece = (lane >> 4) * 32;
  const int n = min(n0 + row, t.N - 1), mr = min(t.m0 + row, t.M - 1);
  const char *a = t.A + (int64_t)mr * p.lda + piece, *b = t.B + (int64_t)n * p.ldb + piece;
  const uint8_t *sa_row = t.sa + (int64_t)mr * p.sa_ld, *sb_row = WIDE ? nullptr : t.sb + (int64_t)(n >> p.sb_shift) * p.sb_ld;
  const float *wide = WIDE ? reinterpret_cast<const float *>(t.sb) + (int64_t)__builtin_amdgcn_readfirstlane(min(n0, t.N - 1) >> 7) * p.sb_ld : nullptr;
  v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int RUN = 2;
  struct Run {
    v4i a[RUN][2], b[RUN][2];
    uint32_t sa, sb;
  };
  const auto request = [&](Run &v, int kb) {  // blocks past the end: the last one, not used
#pragma unroll
    for (int r = 0; r < RUN; ++r) {
      const int64_t k = (int64_t)min(kb + r, t.blocks - 1) * F8_BLOCK;
      v.b[r][0] = *reinterpret_cast<const v4i *>(b + k), v.b[r][1] = *reinterpret_cast<const v4i *>(b + k + 16);
    }
#pragma unroll
    for (int r = 0; r < RUN; ++r) {
      const int64_t k = (int64_t)min(kb + r, t.blocks - 1) * F8_BLOCK;
      v.a[r][0] = *reinterpret_cast<const v4i *>(a + k), v.a[r][1] = *reinterpret_cast<const v4i *>(a + k + 16);
    }
    v.sa = f8_scales(sa_row, t.first + kb, t.readable);
    v.sb = WIDE ? 0x7f7f7f7fu : f8_scales(sb_row, t.first + kb, t.readable);
  };
  const auto multiply = [&](const Run &v, int kb) {
#pragma unroll
    for (int r = 0; r < RUN; ++r) {
      if (kb + r >= t.blocks) break;
      const float fa = __uint_as_float((v.sa >> (8 * r) & 0xffu) << 23), fb = __uint_as_float((v.sb >> (8 * r) & 0xffu) << 23);
      v4f sum = WIDE ? v4f{} : acc;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          v8bf wa, wb;
#pragma unroll
          for (int i = 0; i < 2; ++i) f8_widen(v.a[r][h][c * 2 + i], fa, wa, i * 4), f8_widen(v.b[r][h][c * 2 + i], fb, wb, i * 4);
          sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, wa, sum, 0, 0, 0);
        }
      if constexpr (WIDE) {
        const float s = wide[kb + r];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(sum[i], s, acc[i]);
      } else {
        acc = sum;
      }
    }
  };
  constexpr int STRIDE = SPLIT * RUN;
  int kb = wave % SPLIT * RUN;
  if (kb < t.blocks) {
    Run v[2];
    request(v[0], kb);
    for (;;) {
      if (kb + STRIDE < t.blocks) request(v[1], kb + STRIDE);
      multiply(v[0], kb);
      kb += STRIDE;
      if (kb >= t.blocks) break;
      if (kb + STRIDE < t.blocks) request(v[0], kb + STRIDE);
      multiply(v[1], kb);
      kb += STRIDE;
      if (kb >= t.blocks) break;
    }
  }
  if constexpr (SPLIT > 1) {
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave % SPLIT) return;
#pragma unroll
    for (int w = 1; w < SPLIT; ++w) acc += sums[wave + w][lane];
  }
  const int m = t.m0 + (lane & 15), nn = n0 + (lane >> 4) * 4;
  if (m >= t.M || nn >= t.N) return;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = acc[i] + (p.bias ? p.bias[min(nn + i, t.N - 1)] : 0.0f);
  if (p.type == BNN_BF16) store4(reinterpret_cast<__bf16 *>(t.y) + m * p.ldy, nn, t.N, v);
  else if (p.type == BNN_F16) store4(reinterpret_cast<_Float16 *>(t.y) + m * p.ldy, nn, t.N, v);
  else store4(reinterpret_cast<float *>(t.y) + m * p.ldy, nn, t.N, v);
}
template <int SPLIT, bool WIDE>
__global__ __launch_bounds__(512, 4) void f8_few_kernel(F8Operands p) {
  __shared__ v4f sums[8][64];
  f8_few_product<SPLIT, WIDE>(p, sums);
}

}  // namespace bnn
