// Matrix-core product of 16-bit operands whose k axis runs down the rows of memory, out[m][n] = sum over k of
// A(k, m) * B[k][n] with A in rows of k (the gradient of an input from a weight) or k-major as B is (the gradient of a
// weight from an input): no transposed copy is made, the transposing read of LDS turns rows of k into fragments.
// bf16, 8192 x 4096 by k 16384 and 16384 x 4096 by k 8192: 760 to 800 us one after the other, 1370 to 1450 TFLOP/s, matrix units busy
// 70 % of the cycles; 820 and 870 us in a whole training pass.
#pragma once
#include "tile_mm.h"

namespace bnn {

// k runs over `segments` stretches of K: stretch s reads B0 or B1, and A from s * segA values of k on.
struct KmOperands {
  const char *A, *B0, *B1;
  int64_t lda, ldb;  // bytes between rows
  int64_t segA;
  int M, N, K, segments;
  int tilesM, tilesN, splits;  // the steps of k are dealt out to `splits` workgroups a tile
};

constexpr int KM_STEP = 64;  // values of k a step: 128 bytes of a row of k, or 64 rows

// Where a lane's piece of a row lies, in bytes from a tile's (or a step's) first row.  No sign: 255 rows of 2^24 - 256 bytes, the
// longest that there are (gradients of two projections of 2^22 - 64 values side by side), end 2^24 below 2^32.
__host__ __device__ inline uint32_t km_at(int64_t row, int64_t ld, int64_t within) { return (uint32_t)(row * ld + within); }

// LDS, k-major operand of X columns: rows of 2 X bytes, 16-byte piece c of row k in slot c ^ km_turn(k).  The transposing
// read takes four rows by 16 columns for every 16 lanes; the turns put the eight rows that 32 lanes read on all banks.
template <int X>
__device__ __forceinline__ int km_turn(int k) {
  return X == 64 ? 2 * ((k >> 1 & 1) | (k >> 3 & 1) << 1) : 2 * ((k & 3) | (k >> 3 & 1) << 2);
}

// 16 bytes a lane from base + at straight to LDS at `to`, lane after lane.  Written out: for the builtin the compiler lets
// every transposing read wait for all loads in flight (8192 x 4096 by k 16384, eight waves: 1008 -> 828 us without).  It has no result
// register, and mm_sync, not the compiler, waits for it; m0 takes a wait state before the load reads it.  Nothing else in
// these kernels uses m0 (no builtin load to LDS, no indexed register), so it is not kept.
__device__ __forceinline__ void km_load(const char *base, uint32_t at, uint32_t to) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const v4i res = {(int)(uint32_t)b, (int)((uint32_t)(b >> 32) & 0xffffu), -1, 0x00020000};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(at), "s"(res));
}

template <int TY, int BM, int BN, int WGM, int WGN, int STAGES, bool A_ROWS, class Epilogue>
__device__ __forceinline__ void km_tile_product(const KmOperands &p, const Epilogue &epi, char *lds) {
  using T = MmTraits<TY>;
  using E = typename T::elem;
  using Acc = typename T::acc;
  constexpr int WAVES = WGM * WGN, LOADS_A = BM / 8 / WAVES, LOADS_B = BN / 8 / WAVES, LOADS = LOADS_A + LOADS_B;
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16, STAGE_A = BM * 128, STAGE = (BM + BN) * 128;
  static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && (STAGE & (STAGE - 1)) == 0, "");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  int tm, tn;
  mm_tile(blockIdx.x, p.tilesM, p.tilesN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const float factor = epi.factor();  // requested here: at the end every workgroup would wait for it

  // Offsets of this lane's loads from a step's first value of k.  Rows and columns beyond the operands repeat their last
  // ones, their outputs are not stored; columns come eight at a time (M, if k-major, and N are multiples of eight).
  const auto row_k = [&](int i, auto x) { return (i * WAVES + wave) * (512 / decltype(x)::value) + lane / (decltype(x)::value / 8); };
  const auto columns = [&](int i, auto x, int first, int all) {
    constexpr int X = decltype(x)::value;
    return min(first + (lane % (X / 8) ^ km_turn<X>(row_k(i, x))) * 8, all - 8) * 2;
  };
  using XA = std::integral_constant<int, BM>;
  using XB = std::integral_constant<int, BN>;
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
  uint32_t atA[LOADS_A], atB[LOADS_B];
#pragma unroll
  for (int i = 0; i < LOADS_A; ++i)
    atA[i] = A_ROWS ? km_at(min((i * WAVES + wave) * 8 + (lane >> 3), p.M - 1 - m0), p.lda, piece)
                    : km_at(row_k(i, XA()), p.lda, columns(i, XA(), m0, p.M));
#pragma unroll
  for (int i = 0; i < LOADS_B; ++i) atB[i] = km_at(row_k(i, XB()), p.ldb, columns(i, XB(), n0, p.N));

  const char *const baseA = A_ROWS ? p.A + (int64_t)m0 * p.lda : p.A;
  const int whole = p.K / KM_STEP;  // steps of a stretch
  const auto step_of = [&](int i, const char *&a, const char *&b) {
    const int s = i >= whole ? 1 : 0;
    const int64_t k = (int64_t)(i - s * whole) * KM_STEP, ka = k + s * p.segA;
    a = baseA + (A_ROWS ? 2 * ka : ka * p.lda);
    b = (s ? p.B1 : p.B0) + k * p.ldb;
  };
  const auto request = [&](int i, char *to, int only = -1) {  // all loads of step i, or one
    const char *a, *b;
    step_of(i, a, b);
    const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)to + wave * 1024;
#pragma unroll
    for (int l = 0; l < LOADS; ++l)
      if (only < 0 || l == only) {
        if (l < LOADS_A) km_load(a, atA[l < LOADS_A ? l : 0], dst + l * WAVES * 1024);
        else km_load(b, atB[l < LOADS_A ? 0 : l - LOADS_A], dst + l * WAVES * 1024);
      }
  };

  Acc acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = Acc{0, 0, 0, 0};
  if constexpr (TM * TN == 64)
#pragma unroll
    for (int i = 0; i < TM; ++i) mm_settle(acc[i]);

  // Fragments of 32 values of k.  k-major: lane l of 16 reads four values of row l / 4, and receives column l of four rows.
  const int slot = ((lane >> 4) ^ (lane & 7)) * 16;
  const auto transposing = [&](auto x, int tile) {  // address of this lane in a stage, of 16 columns from 16 * tile on
    constexpr int X = decltype(x)::value;
    const int li = lane & 15, k = (lane >> 4) * 8 + (li >> 2);
    return k * 2 * X + ((tile * 2 ^ km_turn<X>(k)) + (li >> 1 & 1)) * 16 + (li & 1) * 8;
  };
  const int fragA = A_ROWS ? (wm * (BM / WGM) + (lane & 15)) * 128 + slot : transposing(XA(), wm * TM);
  const int fragB = STAGE_A + transposing(XB(), wn * TN);
  struct Half {
    u32x4 a[TM], b[TN];
  };
  typedef short s4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const auto read8 = [&](int at, auto x) {  // rows 4 apart: the same turn
    constexpr int X = decltype(x)::value;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(lds + at)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(lds + at + 8 * X)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  };
  const auto fetch_one = [&](Half &f, int stage, int half, int k) {  // B's first
    const int j = k < TN ? k : 0, i = k < TN ? 0 : k - TN;
    if (k < TN) f.b[j] = read8((stage + fragB ^ j * 32) + half * 64 * BN, XB());
    else if constexpr (A_ROWS) f.a[i] = *reinterpret_cast<const u32x4 *>(lds + (stage + fragA ^ half * 64) + i * 2048);
    else f.a[i] = read8((stage + fragA ^ i * 32) + half * 64 * BM, XA());
  };
  const auto fetch = [&](Half &f, int stage, int half) {
#pragma unroll
    for (int k = 0; k < TM + TN; ++k) fetch_one(f, stage, half, k);
  };
  constexpr bool IN_PLACE = TM * TN == 64;
  const auto nothing = [](int) {};
  const auto multiply = [&](const Half &f) {
    if constexpr (IN_PLACE) {
      mm_weave<T, 0>(f, acc, nothing, nothing);
      return;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = T::mfma(f.b[j], f.a[i], acc[i][j]);  // rows of the result: n
  };
  constexpr int READS = 2 * TN + (A_ROWS ? TM : 2 * TM), PER = TM * TN / READS ? TM * TN / READS : 1;
  const auto interleave = [&](auto loads) {
    constexpr int N = decltype(loads)::value;
#pragma unroll
    for (int i = 0; i < READS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (i < N) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // The loop of mm_tile_product, over this workgroup's share of the whole steps.
  const int all = whole * p.segments, split = blockIdx.y;
  const int from = (int)((int64_t)all * split / p.splits), steps = (int)((int64_t)all * (split + 1) / p.splits) - from;
  // What is left of k in a stretch, with zeros behind it, by the last share: requested first and held, where registers allow.
  const int left = p.K - whole * KM_STEP;
  const bool rest = left > 0 && split == p.splits - 1;
  struct Rest {
    u32x4 a[LOADS_A], b[LOADS_B];
  };
  const auto request_rest = [&](Rest &r, int s) {
    const int64_t k = (int64_t)whole * KM_STEP, ka = k + s * p.segA;
    const char *const a = baseA + (A_ROWS ? 2 * ka : ka * p.lda), *const b = (s ? p.B1 : p.B0) + k * p.ldb;
    const u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int l = 0; l < LOADS_A; ++l) {
      if constexpr (A_ROWS) r.a[l] = bytes16<E>(a + (atA[l] - piece), piece, 2 * left);
      else r.a[l] = row_k(l, XA()) < left ? *reinterpret_cast<const u32x4 *>(a + atA[l]) : none;
    }
#pragma unroll
    for (int l = 0; l < LOADS_B; ++l) r.b[l] = row_k(l, XB()) < left ? *reinterpret_cast<const u32x4 *>(b + atB[l]) : none;
  };
  constexpr bool HELD = BM * BN < 256 * 256;
  Rest held[2];
  if (HELD && rest) {
    request_rest(held[0], 0);
    if (p.segments > 1) request_rest(held[1], 1);
  }
  for (int i = 0; i < min(steps, STAGES); ++i) request(from + i, lds + i * STAGE);
  if (steps) {
    Half first, second;
    if (steps >= STAGES) mm_sync<(STAGES - 1) * LOADS>();
    else mm_sync<0>();
    fetch(first, 0, 0);
    int now = 0;
    const auto turn = [&](int i, auto loads) {
      const int next = now + 1 == STAGES ? 0 : now + 1;
      if constexpr (IN_PLACE) {
        mm_weave<T, TM + TN>(first, acc, [&](int k) { fetch_one(second, now * STAGE, 1, k); }, nothing);
        if (i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
        else mm_sync<0>();
        mm_weave<T, TM + TN>(second, acc, [&](int k) { fetch_one(first, next * STAGE, 0, k); }, [&](int k) {
          if constexpr (decltype(loads)::value > 0)
            if (k < LOADS) request(from + i + STAGES, lds + now * STAGE, k);
        });
        now = next;
        return;
      }
      __builtin_amdgcn_sched_barrier(0);
      fetch(second, now * STAGE, 1);
      multiply(first);
      interleave(std::integral_constant<int, 0>());
      if (i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
      else mm_sync<0>();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (decltype(loads)::value > 0) request(from + i + STAGES, lds + now * STAGE);
      fetch(first, next * STAGE, 0);
      multiply(second);
      interleave(loads);
      now = next;
    };
    int i = 0;
    if constexpr (IN_PLACE) {  // both stages' addresses in registers
      static_assert(STAGES == 2, "");
      for (; i + 1 + STAGES < steps; i += 2) {
        now = 0;
        turn(i, std::integral_constant<int, LOADS>());
        now = 1;
        turn(i + 1, std::integral_constant<int, LOADS>());
      }
      now = 0;
    }
    for (; i + STAGES < steps; ++i) turn(i, std::integral_constant<int, LOADS>());
    for (; i + 1 < steps; ++i) turn(i, std::integral_constant<int, 0>());
    fetch(second, now * STAGE, 1);
    multiply(first);
    multiply(second);
  }
  if (rest) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s >= p.segments) break;
      if (!HELD) request_rest(held[s], s);
      __syncthreads();
#pragma unroll
      for (int l = 0; l < LOADS_A; ++l) *reinterpret_cast<u32x4 *>(lds + (l * WAVES + wave) * 1024 + lane * 16) = held[s].a[l];
#pragma unroll
      for (int l = 0; l < LOADS_B; ++l) *reinterpret_cast<u32x4 *>(lds + STAGE_A + (l * WAVES + wave) * 1024 + lane * 16) = held[s].b[l];
      __syncthreads();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        Half f;
        fetch(f, 0, half);
        multiply(f);
      }
    }
  }

  if constexpr (IN_PLACE)
#pragma unroll
    for (int i = 0; i < TM; ++i) mm_settle(acc[i]);
  const int m = m0 + wm * (BM / WGM) + (lane & 7), n = n0 + wn * (BN / WGN) + (lane & 8) * 2 + (lane >> 4) * 4;
  static_assert(TN % 2 == 0, "");
#pragma unroll
  for (int j = 0; j < TN; j += 2)
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      Acc x[2] = {acc[i][j], acc[i][j + 1]};
      mm_longer(x);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (n + j * 16 < p.N && m + i * 16 + h * 8 < p.M) epi(m + i * 16 + h * 8, n + j * 16, p.N, split, factor, x[h]);
    }
}

template <int TY, int BM, int BN, int WGM, int WGN, int STAGES, bool A_ROWS, class Epilogue>
__global__ __launch_bounds__(64 * WGM *WGN, WGM *WGN / 4) void km_tile_kernel(KmOperands p, Epilogue epi) {
  __shared__ __attribute__((aligned(16))) char lds[STAGES * (BM + BN) * 128];
  km_tile_product<TY, BM, BN, WGM, WGN, STAGES, A_ROWS>(p, epi, lds);
}

template <int TY, int BM, int BN, int WGM, int WGN, int STAGES, bool A_ROWS, class Epilogue>
bnn_status launch_km_tile(KmOperands p, const Epilogue &epi, int kid, hipStream_t s) {
  p.tilesM = (p.M - 1) / BM + 1;
  p.tilesN = (p.N - 1) / BN + 1;
  const int64_t tiles = (int64_t)p.tilesM * p.tilesN;
  if (tiles * 64 * WGM * WGN > 0xffffffffll) return BNN_ERR_UNSUPPORTED;  // threads of a launch
  ProfScope ps(kid, s);
  km_tile_kernel<TY, BM, BN, WGM, WGN, STAGES, A_ROWS, Epilogue><<<dim3((uint32_t)tiles, p.splits), 64 * WGM * WGN, 0, s>>>(p, epi);
  return launch_status();
}

}  // namespace bnn
