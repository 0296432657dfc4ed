// Matrix-core product of two row-major operands, out[m][n] = sum over k of A[m][k] * B[n][k], on 8-bit integers (32-bit
// sums) or 16-bit floating point (fp32 sums), in the form that the quantised and the gated layers share: a workgroup
// computes BM x BN outputs, both operands go through LDS in steps of 128 bytes of k, and an epilogue takes sums of four
// consecutive columns at a time: epi(m, n, N, epi.row(m), epi.columns(n, N), sums..), with n a multiple of 4 below N.
//
// Large products are bound by the matrix units at the clock that they leave the chip (busy 58 to 64 % of the cycles, no bank
// conflicts): 8192^3 in 8 bits 410 to 448 us by card, 2460 to 2680 TOP/s; 8192 x 4096 to 8192 with two weights in bf16 738 to 760 us, 1450 to
// 1490 TFLOP/s.  Small ones by the operands' way into LDS, 25 to 30 bytes a clock and compute unit: 256 x 4096 by 4096 in 8 bits 9 to 10 us.
#pragma once
#include <type_traits>

#include "float_types.h"

namespace bnn {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

enum MmType : int { MM_I8 = 0, MM_BF16 = 1, MM_F16 = 2 };
template <int TY>
struct MmTraits;
template <>
struct MmTraits<MM_I8> {
  using elem = int8_t;
  using acc = v4i;
  static __device__ __forceinline__ acc mfma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(v4i, a), __builtin_bit_cast(v4i, b), c, 0, 0, 0);
  }
  // c in accumulation registers and nowhere else (mm_settle)
  static __device__ __forceinline__ void mfma_in_place(u32x4 a, u32x4 b, acc &c) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  }
};
template <>
struct MmTraits<MM_BF16> {
  using elem = __bf16;
  using acc = v4f;
  static __device__ __forceinline__ acc mfma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  }
  // c in accumulation registers and nowhere else (mm_settle)
  static __device__ __forceinline__ void mfma_in_place(u32x4 a, u32x4 b, acc &c) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  }
};
template <>
struct MmTraits<MM_F16> {
  using elem = _Float16;
  using acc = v4f;
  static __device__ __forceinline__ acc mfma(u32x4 a, u32x4 b, acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
  // c in accumulation registers and nowhere else (mm_settle)
  static __device__ __forceinline__ void mfma_in_place(u32x4 a, u32x4 b, acc &c) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  }
};

// Operands of a product.  DUAL kernels multiply A with two matrices B0 and B1 of N rows each; others have B0 alone.
struct MmOperands {
  const char *A, *B0, *B1;
  int64_t lda, ldb0, ldb1;  // bytes between rows
  int M, N, kbytes;
  int dma;                  // rows and strides are multiples of 16 bytes (mm_dma)
  int tilesM, tilesN;
  int first;                // tile, or group of columns, of this launch's first workgroup: a multiple of eight, or 0
};

// Whether an operand's tiles can go straight to LDS: 16-byte pieces that start on 16 bytes, 32-bit offsets in a tile.
inline bool mm_dma(const void *p, int64_t ld_bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)ld_bytes) & 15u) == 0 && ld_bytes < (1 << 22);
}

// A wave's 64 accumulators of a 128 x 128 tile fill the accumulation registers.  The compiler then has none left to rotate
// them through and copies about 200 of them a step, so these products are written out, each in place.  What the compiler
// does not know of them is waited for here: before the first one reads, and after the last one has written (a matrix
// instruction of eight passes needs eleven wait states before anything else reads its result).
template <class Acc>
__device__ __forceinline__ void mm_settle(Acc (&c)[8]) {
  asm volatile("s_nop 15" : "+a"(c[0]), "+a"(c[1]), "+a"(c[2]), "+a"(c[3]), "+a"(c[4]), "+a"(c[5]), "+a"(c[6]), "+a"(c[7]));
}
// Products of one half step with the next half's reads of LDS between them: first(k) issues the k-th read, second(k) the k-th
// request, if there are so many.
template <class T, int READS, class Half, class Acc, class First, class Second>
__device__ __forceinline__ void mm_weave(const Half &has, Acc (&acc)[8][8], const First &first, const Second &second) {
  constexpr int PER = READS ? 64 / READS : 64;
#pragma unroll
  for (int q = 0; q < 64; ++q) {
    if (q % PER == 0 && q / PER < READS) first(q / PER);
    if (q % 4 == 2) second(q / 4);
    T::mfma_in_place(has.b[q % 8], has.a[q / 8], acc[q / 8][q % 8]);  // rows of the result: n
  }
}

// Two neighbouring tiles of 16 x 16 sums, four columns of row l % 16 a lane, as rows 0 to 7 and 8 to 15 of 16 x 32, row l % 8
// a lane: lanes 8 to 15 of a row of sixteen trade their first tile's sums for the second's of the lanes eight below.  A store
// then covers twice as much of each row: 32 columns of fp32 are a whole cache line (8192 x 4096 to 8192 gated with what its
// backward pass needs 944 -> 861 us, 7039 x 256 to 14336 483 -> 356).
__device__ __forceinline__ void mm_longer(int &a, int &b) {
  const int low = a;
  a = __builtin_amdgcn_update_dpp(a, b, 0x128, 0xf, 0xc, false);  // turned by eight lanes, written in the upper eight
  b = __builtin_amdgcn_update_dpp(b, low, 0x128, 0xf, 0x3, false);  // in the lower eight
}
template <class Acc>
__device__ __forceinline__ void mm_longer(Acc (&x)[2]) {
  if constexpr (sizeof(Acc) % sizeof(int) == 0) {
    constexpr int N = sizeof(Acc) / sizeof(int);
    int a[N], b[N];
    __builtin_memcpy(a, &x[0], sizeof(Acc)), __builtin_memcpy(b, &x[1], sizeof(Acc));
#pragma unroll
    for (int i = 0; i < N; ++i) mm_longer(a[i], b[i]);
    __builtin_memcpy(&x[0], a, sizeof(Acc)), __builtin_memcpy(&x[1], b, sizeof(Acc));
  }  // else of no constants
}

// Tiles in an order in which the workgroups that run at the same time on one XCD (ids go round the eight of them) read few
// different rows: each XCD has a contiguous share of the tiles, and goes through it in bands of 8 tile rows.
__device__ __forceinline__ void mm_tile(int id, int tilesM, int tilesN, int &tm, int &tn) {
  const int total = tilesM * tilesN, xcd = id & 7, share = total >> 3, rest = total & 7;
  const int t = xcd * share + min(xcd, rest) + (id >> 3);
  constexpr int BAND = 8;
  const int band = t / (BAND * tilesN), in = t - band * BAND * tilesN, rows = min(BAND, tilesM - band * BAND);
  tn = in / rows;
  tm = band * BAND + (in - tn * rows);
}

constexpr int MM_STEP = 128;  // bytes of k a step

// All but this wave's last N loads have arrived, its reads of LDS have ended, and every wave of the workgroup is here.
template <int N>
__device__ __forceinline__ void mm_sync() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// This wave's reads and writes of LDS have ended, and every wave of the workgroup is here.
__device__ __forceinline__ void mm_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// LDS: rows of 128 bytes, 16-byte piece c of row r in slot c ^ (r % 8), so that the 16 rows of a fragment spread over all
// banks.  A wave's load fills 8 rows: lane i slot i % 8 of row i / 8.  WGM x WGN waves, each (BM / WGM) x (BN / WGN)
// outputs; with DUAL half of a wave's columns are B0's and half the same columns of B1.
template <int TY, int BM, int BN, int WGM, int WGN, int STAGES, bool DUAL, bool DMA, class Epilogue>
__device__ __forceinline__ void mm_tile_product(const MmOperands &p, const Epilogue &epi, int tm, int tn, char *lds) {
  using T = MmTraits<TY>;
  using E = typename T::elem;
  constexpr int WAVES = WGM * WGN, ROWS = BM + BN, LOADS = ROWS / 8 / WAVES, LOADS_A = BM / 8 / WAVES;
  static_assert(ROWS % (8 * WAVES) == 0 && BM % (8 * WAVES) == 0 && BM % (16 * WGM) == 0 && BN % (16 * WGN * (DUAL ? 2 : 1)) == 0, "");
  constexpr int TM = BM / WGM / 16, TN = BN / WGN / 16, NB = DUAL ? BN / 2 : BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WGN, wn = wave % WGN;
  const int m0 = tm * BM, n0 = tn * NB;
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;  // of the 128 bytes of a step, that this lane's loads bring

  // Where the pieces of this lane's loads come from: rows beyond the operands repeat the last one, their outputs are not
  // stored.
  const char *baseA = p.A + (int64_t)m0 * p.lda, *base0 = p.B0 + (int64_t)n0 * p.ldb0;
  const char *base1 = DUAL ? p.B1 + (int64_t)n0 * p.ldb1 : base0;
  const auto row_of = [&](int i, int64_t &ld) {  // of load i, in its operand's tile
    const int row = (i * WAVES + wave) * 8 + (lane >> 3), nrow = row - BM;
    const bool second = DUAL && nrow >= NB;
    ld = i < LOADS_A ? p.lda : second ? p.ldb1 : p.ldb0;
    return i < LOADS_A ? min(row, p.M - 1 - m0) : min(second ? nrow - NB : nrow, p.N - 1 - n0);
  };
  const auto source = [&](int i) {
    int64_t ld;
    const int r = row_of(i, ld);
    return (i < LOADS_A ? baseA : DUAL && (i * WAVES + wave) * 8 - BM >= NB ? base1 : base0) + r * ld;
  };
  constexpr int STAGE = ROWS * MM_STEP;  // bytes of LDS
  const auto room = [&](char *lds, int i) { return reinterpret_cast<u32x4 *>(lds + (i * WAVES + wave) * 8 * MM_STEP + lane * 16); };

  using Acc = typename T::acc;
  Acc acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = Acc{0, 0, 0, 0};
  if constexpr (TM * TN == 64)
#pragma unroll
    for (int i = 0; i < TM; ++i) mm_settle(acc[i]);

  const int slot = ((lane >> 4) ^ (lane & 7)) * 16;  // of this lane's piece of the first 64 bytes; ^ 64: of the second
  const int fragA = (wm * (BM / WGM) + (lane & 15)) * MM_STEP + slot;
  const int fragB = (BM + wn * (NB / WGN) + (lane & 15)) * MM_STEP + slot;
  struct Half {  // fragments of 64 bytes of k
    u32x4 a[TM], b[TN];
  };
  const auto fetch_one = [&](Half &f, const char *lds, int half, int k) {  // B's first
    const int j = k < TN ? k : 0, i = k < TN ? 0 : k - TN;
    const int row = !DUAL ? j * 16 : j < TN / 2 ? j * 16 : NB + (j - TN / 2) * 16;
    if (k < TN) f.b[j] = *reinterpret_cast<const u32x4 *>(lds + (fragB ^ (half * 64)) + row * MM_STEP);
    else f.a[i] = *reinterpret_cast<const u32x4 *>(lds + (fragA ^ (half * 64)) + i * 16 * MM_STEP);
  };
  const auto fetch = [&](Half &f, const char *lds, int half) {
#pragma unroll
    for (int k = 0; k < TM + TN; ++k) fetch_one(f, lds, half, k);
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
  const auto whole_step = [&](const char *lds) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      Half f;
      fetch(f, lds, half);
      multiply(f);
    }
  };
  // Reads of LDS and requests between matrix instructions, not all in front of them (8192^3 bf16 on eight waves 841 -> 818 us).
  constexpr int PER = TM * TN / (TM + TN) ? TM * TN / (TM + TN) : 1;
  const auto interleave = [&](auto loads) {
    constexpr int N = decltype(loads)::value;
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (i < N) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  const int K = p.kbytes;
  if constexpr (DMA) {
    const auto resA = __builtin_amdgcn_make_buffer_rsrc((void *)baseA, 0, 0xffffffffu, 0x00020000);
    const auto res0 = __builtin_amdgcn_make_buffer_rsrc((void *)base0, 0, 0xffffffffu, 0x00020000);
    const auto res1 = __builtin_amdgcn_make_buffer_rsrc((void *)base1, 0, 0xffffffffu, 0x00020000);
    int at[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      int64_t ld;
      const int r = row_of(i, ld);
      at[i] = (int)(r * ld) + piece;
    }
    constexpr bool BY_LOAD = NB % (8 * WAVES) == 0;  // a load of all waves is of one matrix
    const auto request_one = [&](int i, int k, char *lds) {
      const int row = (i * WAVES + wave) * 8;
      const auto to = (__attribute__((address_space(3))) void *)(lds + row * MM_STEP);
      if (i < LOADS_A) __builtin_amdgcn_raw_ptr_buffer_load_lds(resA, to, 16, at[i], k, 0, 0);
      else if (DUAL && (BY_LOAD ? i * WAVES : i * WAVES + wave) * 8 - BM >= NB) __builtin_amdgcn_raw_ptr_buffer_load_lds(res1, to, 16, at[i], k, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(res0, to, 16, at[i], k, 0, 0);
    };
    const auto request = [&](int k, char *lds) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) request_one(i, k, lds);
    };
    // Both halves of a step's fragments are in registers before the workgroup meets in the middle of the step; from there
    // on its place in LDS takes the step STAGES ahead, and the first half of the next step is read under the products of
    // the second half of this one.
    const int steps = K / MM_STEP;
    // What is left of k after the whole steps, with zeros behind it: requested first and held, where registers allow
    // (1000 x 3001 by k 2321 in 8 bits 18.2 -> 16.5 us), else at the end.
    constexpr bool HELD = BM * BN < 256 * 256;
    const bool rest = steps * MM_STEP < K;
    u32x4 held[LOADS];
    if (HELD && rest) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) held[i] = bytes16<E>(source(i), steps * MM_STEP + piece, K);
    }
    for (int i = 0; i < min(steps, STAGES); ++i) request(i * MM_STEP, lds + i * STAGE);
    if (steps) {
      Half first, second;
      if (steps >= STAGES) mm_sync<(STAGES - 1) * LOADS>();
      else mm_sync<0>();
      fetch(first, lds, 0);
      int now = 0;
      const auto turn = [&](int i, auto loads) {
        const int next = now + 1 == STAGES ? 0 : now + 1;
        if constexpr (IN_PLACE) {
          mm_weave<T, TM + TN>(first, acc, [&](int k) { fetch_one(second, lds + now * STAGE, 1, k); }, nothing);
          if (i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
          else mm_sync<0>();
          mm_weave<T, TM + TN>(second, acc, [&](int k) { fetch_one(first, lds + next * STAGE, 0, k); }, [&](int k) {
            if constexpr (decltype(loads)::value > 0)
              if (k < LOADS) request_one(k, (i + STAGES) * MM_STEP, lds + now * STAGE);
          });
          now = next;
          return;
        }
        __builtin_amdgcn_sched_barrier(0);
        fetch(second, lds + now * STAGE, 1);
        multiply(first);
        interleave(std::integral_constant<int, 0>());
        if (i + STAGES - 1 < steps) mm_sync<(STAGES - 2) * LOADS>();
        else mm_sync<0>();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(loads)::value > 0) {
          request((i + STAGES) * MM_STEP, lds + now * STAGE);
        }
        fetch(first, lds + next * STAGE, 0);
        multiply(second);
        interleave(loads);
        now = next;
      };
      int i = 0;
      for (; i + STAGES < steps; ++i) turn(i, std::integral_constant<int, LOADS>());
      for (; i + 1 < steps; ++i) turn(i, std::integral_constant<int, 0>());
      fetch(second, lds + now * STAGE, 1);
      multiply(first);
      multiply(second);
    }
    if (rest) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < LOADS; ++i) *room(lds, i) = HELD ? held[i] : bytes16<E>(source(i), steps * MM_STEP + piece, K);
      __syncthreads();
      whole_step(lds);
    }
  } else {
    // Two steps in LDS, and the two behind them on their way through registers (four are no faster: the vector caches'
    // rate for pieces that do not start on 16 bytes bounds this form, so large tiles count more).  4096 x 2321 to 4096 gated,
    // bf16: with one step on its way 388 us on 128 x 128 tiles, with two 259, on 256 x 128 221.
    static_assert(STAGES == 2, "");
    const int steps = K / MM_STEP;
    const bool rest = steps * MM_STEP < K;
    const char *src[LOADS];
    u32x4 last[LOADS], held[2][LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) src[i] = source(i);
    if (rest) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) last[i] = bytes16<E>(src[i], steps * MM_STEP + piece, K);
    }
    const auto request = [&](int step, u32x4 (&to)[LOADS]) {  // beyond the last step: that one once more, not used
      const int k = min(step, steps - 1) * MM_STEP + piece;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) to[i] = *reinterpret_cast<const u32x4_any *>(src[i] + k);
    };
    const auto deliver = [&](const u32x4 (&from)[LOADS], char *lds) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) *room(lds, i) = from[i];
    };
    const auto turn = [&](int i, u32x4 (&next)[LOADS], char *now, char *other) {
      mm_meet();  // step i has arrived, and the other half is free
      if (i + 1 < steps) {
        deliver(next, other);
        request(i + 3, next);
      }
      whole_step(now);
    };
    if (steps) {
      request(0, held[0]);
      request(1, held[1]);
      deliver(held[0], lds);
      request(2, held[0]);
      for (int i = 0; i < steps; i += 2) {
        turn(i, held[1], lds, lds + STAGE);
        if (i + 1 < steps) turn(i + 1, held[0], lds + STAGE, lds);
      }
    }
    if (rest) {
      mm_meet();
      deliver(last, lds);
      mm_meet();
      whole_step(lds);
    }
  }

  if constexpr (IN_PLACE)
#pragma unroll
    for (int i = 0; i < TM; ++i) mm_settle(acc[i]);
  constexpr int JT = DUAL ? TN / 2 : TN;
  if constexpr (JT % 2 == 0) {
    const int m = m0 + wm * (BM / WGM) + (lane & 7), n = n0 + wn * (NB / WGN) + (lane & 8) * 2 + (lane >> 4) * 4;
    typename Epilogue::Row rows[TM];  // what the epilogue needs to know of them, all requested at once
#pragma unroll
    for (int i = 0; i < TM; ++i) rows[i] = epi.row(min(m + (lane & 8) + i * 16, p.M - 1));
#pragma unroll
    for (int j = 0; j < JT; j += 2) {
      const int nj = n + j * 16;
      const bool inside = nj < p.N;
      const auto columns = epi.columns(inside ? nj : 0, p.N);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        Acc x[2] = {acc[i][j], acc[i][j + 1]}, y[2];
        typename Epilogue::Row of[2] = {rows[i], rows[i]};
        mm_longer(x);
        mm_longer(of);
        if constexpr (DUAL) {
          y[0] = acc[i][JT + j], y[1] = acc[i][JT + j + 1];
          mm_longer(y);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int mi = m + i * 16 + h * 8;
          if (!inside || mi >= p.M) continue;
          if constexpr (DUAL) epi(mi, nj, p.N, of[h], columns, x[h], y[h]);
          else epi(mi, nj, p.N, of[h], columns, x[h]);
        }
        if constexpr (IN_PLACE) __builtin_amdgcn_sched_barrier(0);  // one pair's registers at a time
      }
    }
  } else {
    const int m = m0 + wm * (BM / WGM) + (lane & 15), n = n0 + wn * (NB / WGN) + (lane >> 4) * 4;
    typename Epilogue::Row rows[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) rows[i] = epi.row(min(m + i * 16, p.M - 1));
#pragma unroll
    for (int j = 0; j < JT; ++j) {
      if (n + j * 16 >= p.N) continue;
      const auto columns = epi.columns(n + j * 16, p.N);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (m + i * 16 >= p.M) continue;
        if constexpr (DUAL) epi(m + i * 16, n + j * 16, p.N, rows[i], columns, acc[i][j], acc[i][JT + j]);
        else epi(m + i * 16, n + j * 16, p.N, rows[i], columns, acc[i][j]);
      }
    }
  }
}

template <int TY, int BM, int BN, int WGM, int WGN, int STAGES, bool DUAL, bool DMA, class Epilogue>
__global__ __launch_bounds__(64 * WGM *WGN, WGM *WGN < 4 ? 1 : WGM *WGN / 4) void mm_tile_kernel(MmOperands p, Epilogue epi) {
  __shared__ __attribute__((aligned(16))) char lds[STAGES * (BM + BN) * MM_STEP];
  int tm, tn;
  mm_tile(p.first + blockIdx.x, p.tilesM, p.tilesN, tm, tn);
  mm_tile_product<TY, BM, BN, WGM, WGN, STAGES, DUAL, DMA>(p, epi, tm, tn, lds);
}

template <int TY, int BM, int BN, int WGM, int WGN, int STAGES, bool DUAL, bool DMA, class Epilogue>
bnn_status launch_mm_tile(MmOperands p, const Epilogue &epi, int kid, hipStream_t s) {
  p.tilesM = (p.M - 1) / BM + 1;
  p.tilesN = (p.N - 1) / (DUAL ? BN / 2 : BN) + 1;
  const int64_t tiles = (int64_t)p.tilesM * p.tilesN;
  if (tiles > 0x7fffffff) return BNN_ERR_UNSUPPORTED;
  ProfScope ps(kid, s);
  wide_launches(tiles, [&](int64_t first, uint32_t n) {
    p.first = (int)first;
    mm_tile_kernel<TY, BM, BN, WGM, WGN, STAGES, DUAL, DMA, Epilogue><<<n, 64 * WGM * WGN, 0, s>>>(p, epi);
  });
  return launch_status();
}

}  // namespace bnn
