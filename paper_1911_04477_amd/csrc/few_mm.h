// The product of tile_mm.h for few rows of A: nothing is reused, the kernel streams B once.
#pragma once
#include "tile_mm.h"

namespace bnn {

// A workgroup owns 16 columns and up to 16 * MT rows; its waves deal the k axis out in runs of 256 bytes, straight from
// memory into matrix operands (any order of k is right as long as both operands have it), and their sums meet in LDS.
template <int TY, int MT, int WAVES, bool DUAL, class Epilogue>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void mm_few_kernel(MmOperands p, Epilogue epi) {
  using T = MmTraits<TY>;
  using E = typename T::elem;
  using Acc = typename T::acc;
  constexpr int NB = DUAL ? 2 : 1, RUN = 4;
  __shared__ Acc sums[WAVES][MT][NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
  const int row = lane & 15, piece = (lane >> 4) * 16;
  const int n = min(n0 + row, p.N - 1);
  const char *b[NB], *a[MT];
  b[0] = p.B0 + n * p.ldb0;
  if constexpr (DUAL) b[1] = p.B1 + n * p.ldb1;
#pragma unroll
  for (int i = 0; i < MT; ++i) a[i] = p.A + (int64_t)min(m0 + i * 16 + row, p.M - 1) * p.lda;

  Acc acc[MT][NB];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int d = 0; d < NB; ++d) acc[i][d] = Acc{0, 0, 0, 0};
  const int K = p.kbytes;
  constexpr int STRIDE = WAVES * RUN * 64;
  for (int k = wave * RUN * 64; k < K; k += STRIDE) {
    u32x4 vb[RUN][NB], va[RUN][MT];
    if (k + RUN * 64 <= K) {
#pragma unroll
      for (int r = 0; r < RUN; ++r) {
#pragma unroll
        for (int d = 0; d < NB; ++d) vb[r][d] = *reinterpret_cast<const u32x4_any *>(b[d] + k + r * 64 + piece);
#pragma unroll
        for (int i = 0; i < MT; ++i) va[r][i] = *reinterpret_cast<const u32x4_any *>(a[i] + k + r * 64 + piece);
      }
    } else {
#pragma unroll
      for (int r = 0; r < RUN; ++r) {
#pragma unroll
        for (int d = 0; d < NB; ++d) vb[r][d] = mm_piece<E>(b[d], k + r * 64 + piece, K);
#pragma unroll
        for (int i = 0; i < MT; ++i) va[r][i] = mm_piece<E>(a[i], k + r * 64 + piece, K);
      }
    }
#pragma unroll
    for (int r = 0; r < RUN; ++r)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int d = 0; d < NB; ++d) acc[i][d] = T::mfma(vb[r][d], va[r][i], acc[i][d]);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int d = 0; d < NB; ++d) sums[wave][i][d][lane] = acc[i][d];
  __syncthreads();
  for (int i = wave; i < MT; i += WAVES) {
    Acc t[NB];
#pragma unroll
    for (int d = 0; d < NB; ++d) {
      t[d] = sums[0][i][d][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) t[d] += sums[w][i][d][lane];
    }
    const int m = m0 + i * 16 + (lane & 15), nn = n0 + (lane >> 4) * 4;
    if (m < p.M && nn < p.N) {
      if constexpr (DUAL) epi(m, nn, p.N, t[0], t[1]);
      else epi(m, nn, p.N, t[0]);
    }
  }
}

template <int TY, int MT, int WAVES, bool DUAL, class Epilogue>
bnn_status launch_mm_few(const MmOperands &p, const Epilogue &epi, int kid, hipStream_t s) {
  const dim3 grid((uint32_t)((p.N - 1) / 16 + 1), (uint32_t)((p.M - 1) / (16 * MT) + 1));
  ProfScope ps(kid, s);
  mm_few_kernel<TY, MT, WAVES, DUAL, Epilogue><<<grid, 64 * WAVES, 0, s>>>(p, epi);
  return launch_status();
}

// Which kernel takes a product: up to 64 rows the one that streams B, else tiles, the large ones where they occupy the
// compute units.
template <int TY, bool DUAL, class Epilogue>
bnn_status run_product(const MmOperands &p, const Epilogue &epi, int kid_few, int kid, hipStream_t s) {
  if (p.M <= 16) return launch_mm_few<TY, 1, 8, DUAL>(p, epi, kid_few, s);
  if (p.M <= 64) return launch_mm_few<TY, 4, 8, DUAL>(p, epi, kid_few, s);
  if (!p.dma) return launch_mm_tile<TY, 128, 128, 2, 2, DUAL, false>(p, epi, kid, s);
  const int64_t large = (int64_t)((p.M - 1) / 256 + 1) * ((p.N - 1) / (DUAL ? 128 : 256) + 1);
  if (large < device_cu_count()) return launch_mm_tile<TY, 128, 128, 2, 2, DUAL, true>(p, epi, kid, s);
  return launch_mm_tile<TY, 256, 256, 2, 4, DUAL, true>(p, epi, kid, s);
}

}  // namespace bnn
