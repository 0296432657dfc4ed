// The product of tile_mm.h for few rows of A: nothing is reused, the kernel streams B once, and is bound by that: one row of
// 4096 to 8192 with two weights in bf16 26 us, 5.1 TB/s; by 4096 x 4096 in 8 bits 4.5 us, 3.7 TB/s, of which 2 are the launch.  Fewer
// than 4096 columns leave units without work (1 x 8192 by 512 in 8 bits 6.2 us).
#pragma once
#include "tile_mm.h"

namespace bnn {

// A workgroup owns 16 columns and up to 16 rows; its waves deal the k axis out in runs of RUN * 64 bytes, straight from
// memory into matrix operands (any order of k is right as long as both operands have it), and their sums meet in LDS.  The
// next run is requested before the products of the present one.
template <int TY, int WAVES, int RUN, bool DUAL, class Epilogue>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void mm_few_kernel(MmOperands p, Epilogue epi) {
  using T = MmTraits<TY>;
  using E = typename T::elem;
  using Acc = typename T::acc;
  constexpr int NB = DUAL ? 2 : 1, BYTES = RUN * 64;
  __shared__ Acc sums[WAVES][NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = (p.first + blockIdx.x) * 16;
  const int row = lane & 15, piece = (lane >> 4) * 16;
  const int n = min(n0 + row, p.N - 1);
  const char *b[NB], *const a = p.A + (int64_t)min(row, p.M - 1) * p.lda;
  b[0] = p.B0 + n * p.ldb0;
  if constexpr (DUAL) b[1] = p.B1 + n * p.ldb1;

  Acc acc[NB];
#pragma unroll
  for (int d = 0; d < NB; ++d) acc[d] = Acc{0, 0, 0, 0};
  struct Run {
    u32x4 b[RUN][NB], a[RUN];
  };
  const int K = p.kbytes;
  const auto request = [&](Run &v, int k) {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
#pragma unroll
      for (int d = 0; d < NB; ++d) v.b[r][d] = *reinterpret_cast<const u32x4_any *>(b[d] + k + r * 64 + piece);
#pragma unroll
    for (int r = 0; r < RUN; ++r) v.a[r] = *reinterpret_cast<const u32x4_any *>(a + k + r * 64 + piece);
  };
  const auto multiply = [&](const Run &v) {
#pragma unroll
    for (int r = 0; r < RUN; ++r)
#pragma unroll
      for (int d = 0; d < NB; ++d) acc[d] = T::mfma(v.b[r][d], v.a[r], acc[d]);
  };
  constexpr int STRIDE = WAVES * BYTES;
  int k = wave * BYTES;
  if (k + BYTES <= K) {
    Run v[2];
    request(v[0], k);
    for (;;) {
      if (k + STRIDE + BYTES <= K) request(v[1], k + STRIDE);
      multiply(v[0]);
      k += STRIDE;
      if (k + BYTES > K) break;
      if (k + STRIDE + BYTES <= K) request(v[0], k + STRIDE);
      multiply(v[1]);
      k += STRIDE;
      if (k + BYTES > K) break;
    }
  }
  for (const int end = min(K, k + BYTES); k < end; k += 64) {  // the last run, cut short
    u32x4 vb[NB];
#pragma unroll
    for (int d = 0; d < NB; ++d) vb[d] = bytes16<E>(b[d], k + piece, K);
    const u32x4 va = bytes16<E>(a, k + piece, K);
#pragma unroll
    for (int d = 0; d < NB; ++d) acc[d] = T::mfma(vb[d], va, acc[d]);
  }
#pragma unroll
  for (int d = 0; d < NB; ++d) sums[wave][d][lane] = acc[d];
  __syncthreads();
  if (wave) return;
  Acc t[NB];
#pragma unroll
  for (int d = 0; d < NB; ++d) {
    t[d] = sums[0][d][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) t[d] += sums[w][d][lane];
  }
  const int m = lane & 15, nn = n0 + (lane >> 4) * 4;
  if (m < p.M && nn < p.N) {
    if constexpr (DUAL) epi(m, nn, p.N, epi.row(m), epi.columns(nn, p.N), t[0], t[1]);
    else epi(m, nn, p.N, epi.row(m), epi.columns(nn, p.N), t[0]);
  }
}

template <int TY, int WAVES, int RUN, bool DUAL, class Epilogue>
bnn_status launch_mm_few(MmOperands p, const Epilogue &epi, int kid, hipStream_t s) {
  ProfScope ps(kid, s);
  wide_launches((p.N - 1) / 16 + 1, [&](int64_t first, uint32_t n) {
    p.first = (int)first;
    mm_few_kernel<TY, WAVES, RUN, DUAL, Epilogue><<<n, 64 * WAVES, 0, s>>>(p, epi);
  });
  return launch_status();
}

// Which kernel takes a product: that of few rows up to 16, else the cheapest by the rounds of tiles that the compute units go through,
// in hundredths of a round of 256 x 256 tiles.  `one`: every unit has one tile at most; `two`: a round of two tiles a unit
// (256 x 256 and 256 x 128: one at a time).  What the small tiles wait for is their operands' way into LDS, so that times
// measured in 8 bits at k 4096 hold for 16 bits at k 2048.  In 8 bits, k 4096, by 4096, us:
//   rows   256x256  256x128  128x128  128x64  64x64  64x32  32x32
//   2048     45       33       35      42      53
//    512              25       17      12.7    15     20     25
//    256              25       17      12       9.8   10.9   12 to 16
//    100              23       15      11.4     9.2    9.1    9.1
//     64              23       15      10.6     8.9    8.7    7.8
struct MmForm {
  int bm, bn, one, two;
};
enum : int { MM_256, MM_256_128, MM_128, MM_128_64, MM_64, MM_64_32, MM_32, MM_FORM_COUNT, MM_128_DEEP = MM_FORM_COUNT, MM_FEW };
constexpr MmForm MM_FORMS[MM_FORM_COUNT] = {{256, 256, 100, 200}, {256, 128, 70, 140}, {128, 128, 45, 74}, {128, 64, 28, 46},
                                            {64, 64, 22, 32},     {64, 32, 19, 28},    {32, 32, 17, 24}};
inline int mm_form(int M, int N, bool dual, bool dma, int64_t units) {
  if (M <= 16) return MM_FEW;
  int best = MM_64;
  int64_t least = INT64_MAX;
  for (int f = 0; f < MM_FORM_COUNT; ++f) {
    if (!dma && f != MM_256_128 && f != MM_128 && f != MM_64) continue;
    const MmForm &t = MM_FORMS[f];
    const int64_t tiles = (int64_t)((M - 1) / t.bm + 1) * ((N - 1) / (dual ? t.bn / 2 : t.bn) + 1);
    const int64_t cost = t.bm == 256 ? (tiles + units - 1) / units * t.one : tiles <= units ? t.one : (tiles + 2 * units - 1) / (2 * units) * t.two;
    if (cost <= least) least = cost, best = f;
  }
  if (best == MM_128 && dma && (int64_t)((M - 1) / 128 + 1) * ((N - 1) / (dual ? 64 : 128) + 1) <= units) return MM_128_DEEP;
  return best;
}

template <int TY, bool DUAL, class Epilogue>
bnn_status run_product(const MmOperands &p, const Epilogue &epi, int kid_few, int kid, hipStream_t s) {
  const int form = mm_form(p.M, p.N, DUAL, p.dma, device_cu_count());
  if (form == MM_FEW) return launch_mm_few<TY, 8, 4, DUAL>(p, epi, kid_few, s);
  if (!p.dma) {  // through registers
    if (form == MM_256_128) return launch_mm_tile<TY, 256, 128, 4, 2, 2, DUAL, false>(p, epi, kid, s);
    if (form == MM_128) return launch_mm_tile<TY, 128, 128, 4, 2, 2, DUAL, false>(p, epi, kid, s);
    return launch_mm_tile<TY, 64, 64, 4, 2, 2, DUAL, false>(p, epi, kid, s);
  }
  switch (form) {
    case MM_256:  // 128 outputs a thread: what the epilogue does is compiled for the call
      return epi.fixed([&](const auto &known) { return launch_mm_tile<TY, 256, 256, 2, 2, 2, DUAL, true>(p, known, kid, s); });
    case MM_256_128: return launch_mm_tile<TY, 256, 128, 4, 2, 3, DUAL, true>(p, epi, kid, s);
    // one tile a unit: four steps ahead (1024 x 4096 by k 1024 in 8 bits 8.9 us, with two 9.6); else two tiles a unit
    // (2048 x 4096 by 4096 35 us, 41 with four steps)
    case MM_128_DEEP: return launch_mm_tile<TY, 128, 128, 2, 4, 4, DUAL, true>(p, epi, kid, s);
    case MM_128: return launch_mm_tile<TY, 128, 128, 4, 2, 2, DUAL, true>(p, epi, kid, s);
    // eight waves a tile where its columns allow: 256 x 4096 by 4096 in 8 bits takes 9.8 us on 64 x 64, with four waves 11.8
    case MM_128_64: return launch_mm_tile<TY, 128, 64, 4, 2, 3, DUAL, true>(p, epi, kid, s);
    case MM_64: return launch_mm_tile<TY, 64, 64, 4, 2, 4, DUAL, true>(p, epi, kid, s);
    case MM_64_32: return launch_mm_tile<TY, 64, 32, 4, 1, 4, DUAL, true>(p, epi, kid, s);
    default: return launch_mm_tile<TY, 32, 32, 2, 1, 6, DUAL, true>(p, epi, kid, s);
  }
}

}  // namespace bnn
