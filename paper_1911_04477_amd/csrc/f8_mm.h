// Matrix-core product of two row-major operands in e4m3 with a scale for each block of 128 values (f8.h),
//   y[m][n] = sum over blocks of scaleA[m][b] * scaleB[n][b] * (sum over the block's k of A[m][k] * B[n][k]),
// fp32 sums.  A step of 128 bytes of k is one block.  Scales that are powers of two go into the matrix instruction as bytes;
// fp32 scales of B, one for 128 rows and a block, multiply a block's sums on the vector unit (the rows' scale is
// in them by then), which fits into the shadow of the matrix instructions: 16 multiply-adds for two of them.
//
// The 8-bit matrix instruction is exact in single products and adds up groups of them in fp32, but within a group of eight it keeps no bits
// below 2^-13 of the largest: measured on normal values, 1.5e-5 of the result in the 2-norm, whatever the length (at worst 2^-10 of the sum of
// magnitudes).  That is a hundredth of what rounding the result to bf16 costs (a fourteenth in fp16), and far below the 2^-4 of the operands'
// own rounding, so results in 16 bits of many rows take it, at twice the rate.  fp32 results, and the kernel of few rows, which memory bounds, are
// EXACT: values go to bf16 on their way into the 16-bit instruction, times their scales; no digit is lost, and sums are fp32's.
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
  int M, N, blocks;
  int tilesM, tilesN;
  int64_t first;     // tile of this launch's first workgroup
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
  char *y;
  int m0, n0, M, N;    // first row and column; the ends
  int blocks;
};

// Tiles of rows by group: the tiles before each group from a scan over the experts' counts (64 at a time; a launch has
// workgroups for as many as there can be, those beyond end).  Returns the number of tiles of rows; finds tile tm's group where
// tm is among them: expert, its first and last row.
struct F8Group {
  int e, lo, hi;
};
__device__ __forceinline__ int f8_clamped(const int32_t *offsets, int e, int S) { return min(max(offsets[e], 0), S); }
template <int BM>
__device__ __forceinline__ int f8_row_tiles(const F8Operands &p, int wanted, F8Group &g, int &tile) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    const int e = e0 + lane;
    const int lo = e < p.E ? f8_clamped(p.offsets, e, p.M) : 0, hi = e < p.E ? max(f8_clamped(p.offsets, e + 1, p.M), lo) : 0;
    int sum = (hi - lo + BM - 1) / BM;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    if (wanted >= 0) {
      const uint64_t past = __ballot(before + sum > wanted);
      if (past) {
        const int l = __builtin_ctzll(past);
        const int start = l ? __shfl(sum, l - 1) : 0;
        g.e = __builtin_amdgcn_readfirstlane(e0 + l);
        g.lo = __builtin_amdgcn_readfirstlane(__shfl(lo, l)), g.hi = __builtin_amdgcn_readfirstlane(__shfl(hi, l));
        tile = __builtin_amdgcn_readfirstlane(wanted - before - start);
        return -1;
      }
    }
    before += __builtin_amdgcn_readfirstlane(__shfl(sum, 63));
  }
  return before;
}

// The tile of a workgroup; false: none is left for it.  BM x BN outputs.
template <int BM, int BN>
__device__ __forceinline__ bool f8_part(const F8Operands &p, int64_t id, F8Part &t) {
  int tm, tn, tile;
  const int size = p.type == BNN_F32 ? 4 : 2, readable = (p.blocks + 3) & ~3;
  if (p.groups == F8_GROUP_ROWS) {
    F8Group g = {0, 0, 0};
    const int tilesM = f8_row_tiles<BM>(p, -1, g, tile);
    if (id >= (int64_t)tilesM * p.tilesN) return false;
    mm_tile((int)id, tilesM, p.tilesN, tm, tn);
    f8_row_tiles<BM>(p, tm, g, tile);
    t = {p.A, p.B + g.e * p.b_es, p.sa, static_cast<const uint8_t *>(p.sb) + g.e * p.sb_es, readable, static_cast<char *>(p.y),
         g.lo + tile * BM, tn * BN, g.hi, p.N, p.blocks};
    return true;
  }
  const int64_t of = (int64_t)p.tilesM * p.tilesN;
  if (p.groups == F8_GROUP_K) {
    const int e = (int)(id / of);
    if (e >= p.E) return false;
    mm_tile((int)(id - e * of), p.tilesM, p.tilesN, tm, tn);
    const int end = p.blocks * F8_BLOCK, lo = f8_clamped(p.offsets, e, end) / F8_BLOCK, hi = max(f8_clamped(p.offsets, e + 1, end) / F8_BLOCK, lo);
    t = {p.A + (int64_t)lo * F8_BLOCK, p.B + (int64_t)lo * F8_BLOCK, p.sa + lo, static_cast<const uint8_t *>(p.sb) + lo,
         readable - lo, static_cast<char *>(p.y) + e * p.y_es * size, tm * BM, tn * BN, p.M, p.N, hi - lo};
    return true;
  }
  if (id >= of) return false;
  mm_tile((int)id, p.tilesM, p.tilesN, tm, tn);
  t = {p.A, p.B, p.sa, static_cast<const uint8_t *>(p.sb), readable, static_cast<char *>(p.y), tm * BM, tn * BN, p.M, p.N, p.blocks};
  return true;
}

// The scales of four blocks of a row from block kb on; past the row's bytes nothing is read.
__device__ __forceinline__ uint32_t f8_scales(const uint8_t *row, int kb, int end) {
  typedef uint32_t u32_any __attribute__((aligned(1)));
  const int at = min(kb, end - 4);
  return *reinterpret_cast<const u32_any *>(row + at) >> (8 * (kb - at));
}

__device__ __forceinline__ void f8_store(const F8Operands &p, const F8Part &t, int m, int n, const float (&v)[8]) {
  if (p.type == BNN_BF16) store8(reinterpret_cast<__bf16 *>(t.y) + m * p.ldy, n, t.N, v);
  else if (p.type == BNN_F16) store8(reinterpret_cast<_Float16 *>(t.y) + m * p.ldy, n, t.N, v);
  else store8(reinterpret_cast<float *>(t.y) + m * p.ldy, n, t.N, v);
}

// Four e4m3 values times 2^p as bf16, both exactly.
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void f8_widen(int four, float scale, v8bf &to, int at) {
  const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true);
  to[at] = lo[0], to[at + 1] = lo[1], to[at + 2] = hi[0], to[at + 3] = hi[1];
}
struct F8Wide {
  v8bf v[4];
  __device__ __forceinline__ F8Wide(const v8i &q, uint32_t scale) {  // the scale in the lowest byte
    const float s = __uint_as_float((scale & 0xffu) << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) f8_widen(q[i], s, v[i / 2], i % 2 * 4);
  }
};

__device__ __forceinline__ v16f f8_mfma(const v8i &a, const v8i &b, const v16f &c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}

// LDS as in tile_mm.h: rows of 128 bytes, 16-byte piece c of row r in slot c ^ (r % 8).  WGM x WGN waves of 32 x 32 blocks.
template <int BM, int BN, int WGM, int WGN, int STAGES, bool WIDE, bool EXACT>  // WIDE: fp32 scales of B
__device__ __forceinline__ void f8_tile_product(const F8Operands &p, char *lds) {
  constexpr int WAVES = WGM * WGN, ROWS = BM + BN, LOADS = ROWS / 8 / WAVES, LOADS_A = BM / 8 / WAVES;
  static_assert(ROWS % (8 * WAVES) == 0 && BM % (8 * WAVES) == 0 && BM % (32 * WGM) == 0 && BN % (32 * WGN) == 0, "");
  constexpr int TM = BM / WGM / 32, TN = BN / WGN / 32, STAGE = ROWS * MM_STEP;
  F8Part t;
  if (!f8_part<BM, BN>(p, p.first + blockIdx.x, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;  // of the 128 bytes of a step, that this lane's loads bring
  const char *baseA = t.A + (int64_t)t.m0 * p.lda, *baseB = t.B + (int64_t)t.n0 * p.ldb;
  const auto resA = __builtin_amdgcn_make_buffer_rsrc((void *)baseA, 0, 0xffffffffu, 0x00020000);
  const auto resB = __builtin_amdgcn_make_buffer_rsrc((void *)baseB, 0, 0xffffffffu, 0x00020000);
  uint32_t at[LOADS];  // rows beyond the operands repeat the last one, their outputs are not stored
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = (i * WAVES + wave) * 8 + (lane >> 3);
    at[i] = i < LOADS_A ? (uint32_t)min(row, t.M - 1 - t.m0) * (uint32_t)p.lda + piece
                        : (uint32_t)min(row - BM, t.N - 1 - t.n0) * (uint32_t)p.ldb + piece;
  }
  const auto request = [&](int step, char *lds) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const auto to = (__attribute__((address_space(3))) void *)(lds + (i * WAVES + wave) * 8 * MM_STEP);
      if (i < LOADS_A) __builtin_amdgcn_raw_ptr_buffer_load_lds(resA, to, 16, at[i], step * MM_STEP, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(resB, to, 16, at[i], step * MM_STEP, 0, 0);
    }
  };
  const int steps = t.blocks;
  for (int i = 0; i < min(steps, STAGES); ++i) request(i, lds + i * STAGE);

  // Scales: four blocks' bytes of a row at once, the present block's in the lowest.
  const int row_a = t.m0 + wm * (BM / WGM) + (lane & 31), row_b = t.n0 + wn * (BN / WGN) + (lane & 31);
  const uint8_t *rowsA[TM], *rowsB[WIDE ? 1 : TN];
  uint32_t sa[TM], sb[TN], next_sa[TM], next_sb[TN];
  const float *wide[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) rowsA[i] = t.sa + (int64_t)min(row_a + i * 32, t.M - 1) * p.sa_ld, sa[i] = next_sa[i] = 0u;
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int n = min(t.n0 + wn * (BN / WGN) + j * 32, t.N - 1);  // of the first of 32 columns, which share an fp32 scale
    if constexpr (WIDE) wide[j] = reinterpret_cast<const float *>(t.sb) + (int64_t)__builtin_amdgcn_readfirstlane(n >> 7) * p.sb_ld;
    else rowsB[j] = t.sb + (int64_t)(min(row_b + j * 32, t.N - 1) >> p.sb_shift) * p.sb_ld;
    sb[j] = WIDE ? 127u : 0u, next_sb[j] = sb[j];
  }
  const auto request_scales = [&](int kb) {
#pragma unroll
    for (int i = 0; i < TM; ++i) next_sa[i] = f8_scales(rowsA[i], kb, t.readable);
    if constexpr (!WIDE)
#pragma unroll
      for (int j = 0; j < TN; ++j) next_sb[j] = f8_scales(rowsB[j], kb, t.readable);
  };
  if (steps) request_scales(0);

  v16f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v16f{};
  // Lanes 0 to 31 have pieces 0, 1 of a half step's four, the others 2, 3.
  const int slot = (((lane >> 5) * 2) ^ (lane & 7)) * 16;
  const int fragA = (wm * (BM / WGM) + (lane & 31)) * MM_STEP + slot, fragB = (BM + wn * (BN / WGN) + (lane & 31)) * MM_STEP + slot;
  struct Half {
    v8i a[TM], b[TN];
  };
  const auto read = [&](const char *at) {
    return __builtin_shufflevector(*reinterpret_cast<const v4i *>(at), *reinterpret_cast<const v4i *>(lds + ((at - lds) ^ 16)), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const auto fetch = [&](Half &f, int stage, int half) {
#pragma unroll
    for (int j = 0; j < TN; ++j) f.b[j] = read(lds + stage * STAGE + ((fragB + j * 32 * MM_STEP) ^ (half * 64)));
#pragma unroll
    for (int i = 0; i < TM; ++i) f.a[i] = read(lds + stage * STAGE + ((fragA + i * 32 * MM_STEP) ^ (half * 64)));
  };
  int now = 0;
  for (int i = 0; i < steps; ++i) {
    // (this wave's loads of step i; the rest may be under way)
    if (i + STAGES - 1 < steps) mm_sync<(STAGES - 1) * LOADS>();
    else mm_sync<0>();
    if ((i & 3) == 0) {
#pragma unroll
      for (int k = 0; k < TM; ++k) sa[k] = next_sa[k];
#pragma unroll
      for (int k = 0; k < TN; ++k) sb[k] = next_sb[k];
    }
    Half f[2];
    fetch(f[0], now, 0);
    fetch(f[1], now, 1);
    if constexpr (EXACT) {
      v16f part[TM][TN];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int a = 0; a < TM; ++a) {
          const F8Wide wa(f[h].a[a], sa[a]);
#pragma unroll
          for (int b = 0; b < TN; ++b) {
            const F8Wide wb(f[h].b[b], sb[b]);
            v16f sum = !WIDE ? acc[a][b] : h ? part[a][b] : v16f{};
#pragma unroll
            for (int c = 0; c < 4; ++c) sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb.v[c], wa.v[c], sum, 0, 0, 0);
            (WIDE ? part : acc)[a][b] = sum;
          }
        }
      }
      if constexpr (WIDE) {
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
          for (int b = 0; b < TN; ++b) {
            const float s = wide[b][i];
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = fmaf(part[a][b][r], s, acc[a][b][r]);
          }
      }
    }
    if constexpr (!EXACT)
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
      for (int b = 0; b < TN; ++b) {
        if constexpr (WIDE) {
          v16f part = f8_mfma(f[0].b[b], f[0].a[a], v16f{}, sb[b], sa[a]);
          part = f8_mfma(f[1].b[b], f[1].a[a], part, sb[b], sa[a]);
          const float s = wide[b][i];
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[a][b][r] = fmaf(part[r], s, acc[a][b][r]);
        } else {
          acc[a][b] = f8_mfma(f[0].b[b], f[0].a[a], acc[a][b], sb[b], sa[a]);  // rows of the result: n
          acc[a][b] = f8_mfma(f[1].b[b], f[1].a[a], acc[a][b], sb[b], sa[a]);
        }
      }
#pragma unroll
    for (int k = 0; k < TM; ++k) sa[k] >>= 8;
    if constexpr (!WIDE)
#pragma unroll
      for (int k = 0; k < TN; ++k) sb[k] >>= 8;
    if (i + STAGES < steps) {
      mm_meet();
      request(i + STAGES, lds + now * STAGE);
    }
    if ((i & 3) == 0 && i + 4 < steps) request_scales(i + 4);
    now = now + 1 == STAGES ? 0 : now + 1;
  }

  // A lane has column m = lane % 32 of the blocks and four times four consecutive n, those of lanes 32 above in between: these trade,
  // so that a lane has eight consecutive ones.
  const int m = t.m0 + wm * (BM / WGM) + (lane & 31);
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      const int n = t.n0 + wn * (BN / WGN) + j * 32 + q * 8 + (lane >> 5) * 8;
      float bias[8] = {};
      if (p.bias && n < t.N) load8(bias, p.bias, n, t.N);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        float v[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][q * 4 + r]), __float_as_uint(acc[i][j][q * 4 + 4 + r]), false, false);
          v[r] = __uint_as_float(two[0]) + bias[r], v[4 + r] = __uint_as_float(two[1]) + bias[4 + r];
        }
        if (m + i * 32 < t.M && n < t.N) f8_store(p, t, m + i * 32, n, v);
      }
    }
}

template <int BM, int BN, int WGM, int WGN, int STAGES, bool WIDE, bool EXACT>
__global__ __launch_bounds__(64 * WGM *WGN, WGM *WGN < 4 ? 1 : WGM *WGN / 4) void f8_tile_kernel(F8Operands p) {
  __shared__ __attribute__((aligned(16))) char lds[STAGES * (BM + BN) * MM_STEP];
  f8_tile_product<BM, BN, WGM, WGN, STAGES, WIDE, EXACT>(p, lds);
}

// At most 16 rows of A (of a group): nothing is reused, B is streamed once and bounds the kernel.  A workgroup owns 16
// columns; its waves deal k out in runs of four blocks, straight from memory into registers, and sums meet in LDS.
template <int WAVES, bool WIDE>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void f8_few_kernel(F8Operands p) {
  __shared__ v4f sums[WAVES][64];
  F8Part t;
  if (!f8_part<16, 16>(p, p.first + blockIdx.x, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = lane & 15, piece = (lane >> 4) * 32;
  const int n = min(t.n0 + row, t.N - 1), mr = min(t.m0 + row, t.M - 1);
  const char *a = t.A + (int64_t)mr * p.lda + piece, *b = t.B + (int64_t)n * p.ldb + piece;
  const uint8_t *sa_row = t.sa + (int64_t)mr * p.sa_ld, *sb_row = WIDE ? nullptr : t.sb + (int64_t)(n >> p.sb_shift) * p.sb_ld;
  const float *wide = WIDE ? reinterpret_cast<const float *>(t.sb) + (int64_t)__builtin_amdgcn_readfirstlane(t.n0 >> 7) * p.sb_ld : nullptr;
  v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
  struct Run {
    v4i a[4][2], b[4][2];
    uint32_t sa, sb;
  };
  const auto request = [&](Run &v, int kb) {  // blocks past the end: the last one, not used
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t k = (int64_t)min(kb + r, t.blocks - 1) * F8_BLOCK;
      v.b[r][0] = *reinterpret_cast<const v4i *>(b + k), v.b[r][1] = *reinterpret_cast<const v4i *>(b + k + 16);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t k = (int64_t)min(kb + r, t.blocks - 1) * F8_BLOCK;
      v.a[r][0] = *reinterpret_cast<const v4i *>(a + k), v.a[r][1] = *reinterpret_cast<const v4i *>(a + k + 16);
    }
    v.sa = f8_scales(sa_row, kb, t.readable);
    v.sb = WIDE ? 0x7f7f7f7fu : f8_scales(sb_row, kb, t.readable);
  };
  const auto multiply = [&](const Run &v, int kb) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
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
  constexpr int STRIDE = WAVES * 4;
  int kb = wave * 4;
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
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) acc += sums[w][lane];
  const int m = t.m0 + (lane & 15), nn = t.n0 + (lane >> 4) * 4;
  if (m >= t.M || nn >= t.N) return;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = acc[i] + (p.bias ? p.bias[min(nn + i, t.N - 1)] : 0.0f);
  if (p.type == BNN_BF16) store4(reinterpret_cast<__bf16 *>(t.y) + m * p.ldy, nn, t.N, v);
  else if (p.type == BNN_F16) store4(reinterpret_cast<_Float16 *>(t.y) + m * p.ldy, nn, t.N, v);
  else store4(reinterpret_cast<float *>(t.y) + m * p.ldy, nn, t.N, v);
}

}  // namespace bnn
