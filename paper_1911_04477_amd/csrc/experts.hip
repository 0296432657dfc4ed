// Tokens sorted by expert and back (bnn_expert_sort, bnn_expert_gather, bnn_expert_combine, bnn_expert_combine_backward).  Every
// kernel here moves each value once and is bound by memory, or by its launch.  No atomics on values: sums run over a token's
// experts in their order, and the sort is stable, so calls repeat bit for bit.
#include <algorithm>

#include "rows.h"

namespace bnn {

constexpr int SORT_EXPERTS = 1024, SORT_MOST_BLOCKS = 256, SORT_ONE = 4096;

struct SortParams {
  const void *experts;
  int wide;  // 64-bit indices
  int n, E, align, S;
  int blocks, chunk;  // workgroups, slots of each
  int32_t *counts;    // [blocks, E], blocks > 1
  int32_t *offsets, *rows, *places;
  __device__ __forceinline__ int expert(int slot) const {  // E where there is none
    const int64_t e = wide ? static_cast<const int64_t *>(experts)[slot] : static_cast<const int32_t *>(experts)[slot];
    return e >= 0 && e < E ? (int)e : E;
  }
};

// The lanes of a wave that have the same value: one vote for each of its bits.
__device__ __forceinline__ uint64_t same_lanes(int v, int bits) {
  uint64_t mask = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((v >> b) & 1);
    mask &= (v >> b) & 1 ? set : ~set;
  }
  return mask;
}

// Goes through a wave's slots in order, 64 at a time: f(slot, expert, lanes with the same expert).
template <class F>
__device__ __forceinline__ void sort_walk(const SortParams &p, int begin, int end, int bits, const F &f) {
  const int lane = threadIdx.x & 63;
  for (int s = begin; s < end; s += 64) {
    const int slot = s + lane;
    const int e = slot < end ? p.expert(slot) : p.E;
    f(slot, e, same_lanes(slot < end ? e : p.E + 1, bits));
  }
}
// A wave's share of the workgroup's slots, in whole 64s.
__device__ __forceinline__ void sort_share(const SortParams &p, int &begin, int &end) {
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, first = blockIdx.x * p.chunk, last = min(first + p.chunk, p.n);
  const int each = ((last - first + waves - 1) / waves + 63) & ~63;
  begin = min(first + wave * each, last), end = min(begin + each, last);
}

__global__ __launch_bounds__(1024) void sort_count_kernel(SortParams p) {
  __shared__ int counts[SORT_EXPERTS];
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) counts[e] = 0;
  __syncthreads();
  int begin, end;
  sort_share(p, begin, end);
  const int bits = 32 - __builtin_clz(p.E + 1), lane = threadIdx.x & 63;
  sort_walk(p, begin, end, bits, [&](int, int e, uint64_t same) {
    if (e < p.E && __builtin_ctzll(same) == lane) atomicAdd(&counts[e], __popcll(same));  // whole numbers: any order
  });
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.counts[(int64_t)blockIdx.x * p.E + e] = counts[e];
}

// Each workgroup adds up the others' counts (at most 256 of them), finds where its own slots of every expert begin, and
// places them: a wave's first slot of an expert comes behind those of the waves before it.  Bound by the latency of its passes: 8 slots 3.5 us,
// 3000 7.9, 32768 in 32 workgroups 6.6 and 4.8 for the counts (8192 slots in one workgroup 16, in two launches 10: SORT_ONE).
__global__ __launch_bounds__(1024) void sort_place_kernel(SortParams p) {
  extern __shared__ int words[];  // [waves][E] counts, then positions; [E] total, [E] before, [E + 1] offsets, [16] sums
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, E = p.E, threads = blockDim.x;
  int *const at = words, *const total = at + waves * E, *const before = total + E, *const offsets = before + E, *const sums = offsets + E + 1;
  for (int i = threadIdx.x; i < (waves + 2) * E; i += threads) words[i] = 0;
  __syncthreads();
  int begin, end;
  sort_share(p, begin, end);
  const int bits = 32 - __builtin_clz(E + 1);
  int *const mine = at + wave * E;
  sort_walk(p, begin, end, bits, [&](int, int e, uint64_t same) {
    if (e < E && __builtin_ctzll(same) == lane) mine[e] += __popcll(same);
  });
  if (p.blocks > 1) {
    for (int i = threadIdx.x; i < p.blocks * E; i += threads) {
      const int b = i / E, e = i - b * E, v = p.counts[i];
      if (v) {
        atomicAdd(&total[e], v);
        if (b < (int)blockIdx.x) atomicAdd(&before[e], v);
      }
    }
  }
  __syncthreads();
  if (p.blocks == 1) {
    for (int e = threadIdx.x; e < E; e += threads) {
      int v = 0;
      for (int w = 0; w < waves; ++w) v += at[w * E + e];
      total[e] = v;
    }
    __syncthreads();
  }
  // offsets: a scan over the experts' counts in whole `align`s
  int base = 0;
  for (int e0 = 0; e0 < E; e0 += threads) {
    const int e = e0 + threadIdx.x;
    const int own = e < E ? (total[e] + p.align - 1) / p.align * p.align : 0;
    int sum = own;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < waves; ++w) {
      if (w == wave) sum += all;
      all += sums[w];
    }
    if (e < E) offsets[e] = base + sum - own;
    base += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) offsets[E] = base;
  for (int e = threadIdx.x; e < E; e += threads) {
    int v = offsets[e] + before[e];
    for (int w = 0; w < waves; ++w) {
      const int n = at[w * E + e];
      at[w * E + e] = v;
      v += n;
    }
  }
  __syncthreads();
  sort_walk(p, begin, end, bits, [&](int slot, int e, uint64_t same) {
    const int first = e < E ? mine[e] : 0;
    __builtin_amdgcn_wave_barrier();
    if (e < E) {
      const int pos = first + __popcll(same & ((1ull << lane) - 1));
      if (pos < p.S) p.rows[pos] = slot;
      p.places[slot] = pos;
      if (__builtin_ctzll(same) == lane) mine[e] = first + __popcll(same);
    } else if (slot < end) {
      p.places[slot] = -1;
    }
    __builtin_amdgcn_wave_barrier();
  });
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= E; e += threads) p.offsets[e] = offsets[e];
  // positions without a slot: -1 inside the experts' rows, -2 behind the last
  if (p.align > 1)
    for (int e = blockIdx.x; e < E; e += p.blocks)
      for (int i = offsets[e] + total[e] + threadIdx.x; i < min(offsets[e + 1], p.S); i += threads) p.rows[i] = -1;
  for (int64_t i = (int64_t)offsets[E] + blockIdx.x * threads + threadIdx.x; i < p.S; i += (int64_t)p.blocks * threads) p.rows[i] = -2;
}

struct GatherParams {
  const char *x;
  char *y;
  int64_t x_ld, y_ld;  // bytes
  const int32_t *rows;
  FastDiv k;
  int64_t slots, S, chunks;
  int bytes, size;
};

// A wave takes 4 KB of a row, four 16-byte pieces a lane, all loads first, and writes past the caches (8192 tokens to four experts each, 4096
// wide bf16: 298 MB out, 81 us; two or eight pieces, or ordinary stores, take as long).
constexpr int GATHER_PIECES = 4, GATHER_BYTES = GATHER_PIECES * 64 * 16;
__global__ __launch_bounds__(256) void expert_gather_kernel(GatherParams p) {
  const int64_t id = wide_block() * 4 + (threadIdx.x >> 6);
  const int64_t pos = id / p.chunks;
  if (pos >= p.S) return;
  const int r = __builtin_amdgcn_readfirstlane(p.rows[pos]);
  if (r < -1 || r >= p.slots) return;
  const int lane = threadIdx.x & 63, start = (int)(id - pos * p.chunks) * GATHER_BYTES + lane * 16;
  char *y = p.y + pos * p.y_ld;
  const char *x = r < 0 ? nullptr : p.x + (int64_t)fdiv((uint32_t)r, p.k) * p.x_ld;
  if (p.bytes < 16) {  // by elements of `size` bytes
    const int at = lane * p.size;
    if (at >= p.bytes) return;
    if (p.size == 2) *reinterpret_cast<uint16_t *>(y + at) = x ? *reinterpret_cast<const uint16_t *>(x + at) : 0;
    else *reinterpret_cast<uint32_t *>(y + at) = x ? *reinterpret_cast<const uint32_t *>(x + at) : 0u;
    return;
  }
  u32x4 v[GATHER_PIECES];
  int at[GATHER_PIECES];  // a row's last piece ends with the row: some bytes are copied twice
#pragma unroll
  for (int i = 0; i < GATHER_PIECES; ++i) at[i] = min(start + i * 1024, p.bytes - 16), v[i] = u32x4{0u, 0u, 0u, 0u};
  if (x) {
#pragma unroll
    for (int i = 0; i < GATHER_PIECES; ++i) v[i] = *reinterpret_cast<const u32x4_any *>(x + at[i]);
  }
#pragma unroll
  for (int i = 0; i < GATHER_PIECES; ++i)
    if (start + i * 1024 < p.bytes) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4_any *>(y + at[i]));
}

struct CombineParams {
  const void *ys;
  void *out;
  int64_t ys_ld, out_ld;
  const int32_t *places;
  const float *weights;
  int64_t T, S, chunks;
  int k, D;
};

// A wave takes 512 columns of a token, eight experts' rows requested at once, or 1024 and four.  Bound by memory (8192 tokens of four experts,
// 4096 wide bf16, 336 MB: 65 to 79 us, 4.3 to 5.2 TB/s), for one token by the latency of its three loads, one after the other (2.9 us).
template <class E, int EDGE, int NV>
__global__ __launch_bounds__(256) void expert_combine_kernel(CombineParams p) {
  const int64_t id = wide_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = id / p.chunks;
  if (t >= p.T) return;
  const int c = (int)(id - t * p.chunks) * (512 * NV) + (threadIdx.x & 63) * 8;
  const int32_t *places = p.places + t * p.k;
  const float *weights = p.weights ? p.weights + t * p.k : nullptr;
  float sum[NV][8] = {};
  constexpr int ROWS = NV == 1 ? 8 : 4;
  for (int j0 = 0; j0 < p.k; j0 += ROWS) {
    Piece8<E> v[ROWS][NV];
    float w[ROWS];
    bool has[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      const int jj = min(j0 + j, p.k - 1), pos = places[jj];
      has[j] = j0 + j < p.k && pos >= 0 && pos < p.S;
      w[j] = weights ? weights[jj] : 1.0f;
      if (has[j])
#pragma unroll
        for (int i = 0; i < NV; ++i) v[j][i].load(static_cast<const E *>(p.ys) + pos * p.ys_ld, Place8<EDGE>(c + i * 512, p.D), p.D);
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      if (!has[j]) continue;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Place8<EDGE> at(c + i * 512, p.D);
        if (at.shift) v[j][i].settle(at);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[i][e] = fmaf(w[j], (float)v[j][i].v[e], sum[i][e]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (c + i * 512 < p.D) store8(static_cast<E *>(p.out) + t * p.out_ld, c + i * 512, p.D, sum[i]);
}

struct CombineBackwardParams {
  const void *ys, *dout;
  void *dys;
  int64_t ys_ld, dout_ld, dys_ld;
  const int32_t *rows, *places;
  const float *weights;
  float *dweights;
  int64_t T, S;
  int k, D;
};

// A token a team (a wave, or BLOCK a workgroup); its gradient stays in registers while it goes out to its experts' rows, times
// their weights, and is multiplied with theirs, four experts at a time.  Behind the tokens' workgroups come those that clear the
// rows between the experts' parts, 64 positions each.  Bound by memory (8192 tokens of four experts, 4096 wide bf16, 634 MB: 125 us, 5.1 TB/s).
template <class E, bool BLOCK, int MAXT, int NV, int EDGE>
__global__ __launch_bounds__(MAXT) void combine_backward_kernel(CombineBackwardParams p) {
  __shared__ uint32_t lds[2][4 * 16];
  const int threads = BLOCK ? blockDim.x : 64, tid = BLOCK ? threadIdx.x : threadIdx.x & 63;
  const int64_t tokens = BLOCK ? p.T : (p.T + 3) / 4, block = wide_block();
  if (block >= tokens) {
    if (!p.dys) return;  // nothing to clear: left over in a grid of more than 2^20 workgroups (wide_grid)
    const int64_t first = (block - tokens) * 64, own = first + (threadIdx.x & 63);
    const float none[8] = {};
    for (uint64_t left = __ballot(own < p.S && p.rows[min(own, p.S - 1)] == -1); left; left &= left - 1) {  // one look at all 64
      const int64_t i = first + __builtin_ctzll(left);
      for (int c = threadIdx.x * 8; c < p.D; c += blockDim.x * 8) store8(static_cast<E *>(p.dys) + i * p.dys_ld, c, p.D, none);
    }
    return;
  }
  if constexpr (BLOCK) {
    for (int i = threadIdx.x; i < 128; i += blockDim.x) lds[i >> 6][i & 63] = 0u;
    __syncthreads();
  }
  const int64_t t = BLOCK ? block : block * 4 + (threadIdx.x >> 6);
  if (t >= p.T) return;  // whole waves, without barriers
  Piece8<E> x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) x[i].load(static_cast<const E *>(p.dout) + t * p.dout_ld, Place8<EDGE>((i * threads + tid) * 8, p.D), p.D);
  float d[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place8<EDGE> at((i * threads + tid) * 8, p.D);
    if (at.shift) x[i].settle(at);
#pragma unroll
    for (int e = 0; e < 8; ++e) d[i][e] = (float)x[i].v[e];
  }
  const int32_t *places = p.places + t * p.k;
  int turn = 0;
  for (int j0 = 0; j0 < p.k; j0 += 4) {
    float dot[4] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * threads + tid) * 8;
      const Place8<EDGE> at(c, p.D);
      Piece8<E> y[4];
      int pos[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pos[j] = j0 + j < p.k ? places[j0 + j] : -1;
        if (pos[j] >= p.S) pos[j] = -1;
        if (p.dweights && pos[j] >= 0) y[j].load(static_cast<const E *>(p.ys) + pos[j] * p.ys_ld, at, p.D);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (pos[j] < 0) continue;
        const float w = p.weights ? p.weights[t * p.k + j0 + j] : 1.0f;
        if (p.dys) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = w * d[i][e];
          if (c < p.D) store8(static_cast<E *>(p.dys) + pos[j] * p.dys_ld, c, p.D, v);
        }
        if (p.dweights) {
          if (at.shift) y[j].settle(at);
#pragma unroll
          for (int e = 0; e < 8; ++e) dot[j] = fmaf(d[i][e], (float)y[j].v[e], dot[j]);
        }
      }
    }
    if (!p.dweights) continue;
    team_sum<BLOCK>(dot, lds[turn]);
    turn ^= 1;  // the words of the sums before may still be read
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (tid == 0 && j0 + j < p.k) p.dweights[t * p.k + j0 + j] = dot[j];
  }
}

int64_t expert_capacity(int64_t n, int64_t E, int64_t align) { return (n + std::min(n, E) * (align - 1)) / align * align; }

}  // namespace bnn

extern "C" int64_t bnn_expert_rows(int64_t T, int64_t k, int64_t experts, int64_t align) {
  if (T <= 0 || k <= 0 || experts <= 0 || align <= 0 || align > 4096 || k > (1 << 30) / T || experts > bnn::SORT_EXPERTS) return 0;
  return bnn::expert_capacity(T * k, experts, align);
}

extern "C" size_t bnn_expert_sort_workspace_bytes(int64_t T, int64_t k, int64_t experts) {
  if (T <= 0 || k <= 0 || experts <= 0 || experts > bnn::SORT_EXPERTS || k > (1 << 30) / T || T * k <= bnn::SORT_ONE) return 0;
  return (size_t)bnn::SORT_MOST_BLOCKS * (size_t)experts * 4;
}

extern "C" bnn_status bnn_expert_sort(const void *experts, int index_bytes, int64_t T, int64_t k, int64_t E, int64_t align, int64_t S,
                                      int32_t *offsets, int32_t *rows, int32_t *places, void *workspace, size_t workspace_bytes,
                                      void *stream) {
  using namespace bnn;
  if (T < 0 || k < 1 || E < 1 || align < 1 || S < 0 || (index_bytes != 4 && index_bytes != 8)) return BNN_ERR_SHAPE;
  if (E > SORT_EXPERTS || align > 4096 || k > (1 << 30) || (T > 0 && k > (1 << 30) / T)) return BNN_ERR_UNSUPPORTED;
  const int64_t n = T * k;
  if (S > INT32_MAX || expert_capacity(n, E, align) > INT32_MAX - 4096) return BNN_ERR_UNSUPPORTED;
  if (S < expert_capacity(n, E, align)) return BNN_ERR_SHAPE;
  if (!offsets || (S > 0 && !rows) || (n > 0 && (!experts || !places))) return BNN_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(experts) & (index_bytes - 1)) || !aligned4(offsets) || !aligned4(rows) || !aligned4(places)) return BNN_ERR_ALIGN;
  SortParams p = {experts, index_bytes == 8, (int)n, (int)E, (int)align, (int)S, 1, (int)n, static_cast<int32_t *>(workspace), offsets, rows, places};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int threads = n <= 64 ? 64 : n <= 256 ? 256 : E > 512 ? 512 : 1024;  // LDS: the waves' counts of all experts
  if (n > SORT_ONE) {
    if (workspace_bytes < bnn_expert_sort_workspace_bytes(T, k, E)) return BNN_ERR_WORKSPACE;
    if (!workspace) return BNN_ERR_NULL;
    if (!aligned16(workspace)) return BNN_ERR_ALIGN;
    p.chunk = (int)std::max<int64_t>(1024, ((n - 1) / SORT_MOST_BLOCKS + 1024) / 1024 * 1024);
    p.blocks = (int)((n - 1) / p.chunk + 1);
    ProfScope ps(KID_EXPERT_SORT, s);
    sort_count_kernel<<<p.blocks, threads, 0, s>>>(p);
  }
  const int waves = threads / 64;
  ProfScope ps(KID_EXPERT_SORT, s);
  sort_place_kernel<<<p.blocks, threads, ((waves + 3) * E + 1 + 16) * sizeof(int), s>>>(p);
  return launch_status();
}

extern "C" bnn_status bnn_expert_gather(const void *x, int type, int64_t T, int64_t x_ld, const int32_t *rows, int64_t k, int64_t S,
                                        int64_t D, void *xs, int64_t xs_ld, void *stream) {
  using namespace bnn;
  if (T < 0 || S < 0 || D <= 0 || k < 1 || !float_type(type)) return BNN_ERR_SHAPE;
  if (x_ld < D || xs_ld < D) return BNN_ERR_STRIDE;
  if (S > INT32_MAX || D > (1 << 28) || k > (1 << 30) || (T > 0 && k > (1 << 30) / T)) return BNN_ERR_UNSUPPORTED;
  if (S == 0) return BNN_OK;
  if ((T > 0 && !x) || !rows || !xs) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned4(rows) || !aligned16(xs)) return BNN_ERR_ALIGN;
  const int size = float_size(type);
  GatherParams p = {static_cast<const char *>(x), static_cast<char *>(xs), x_ld * size, xs_ld * size, rows, FastDiv((uint32_t)k), T * k, S, 0,
                    (int)D * size, size};
  p.chunks = (p.bytes - 1) / GATHER_BYTES + 1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_EXPERT_GATHER, s);
  expert_gather_kernel<<<wide_grid((S * p.chunks - 1) / 4 + 1), 256, 0, s>>>(p);
  return launch_status();
}

extern "C" bnn_status bnn_expert_combine(const void *ys, int type, int64_t S, int64_t ys_ld, const int32_t *places, const float *weights,
                                         int64_t T, int64_t k, int64_t D, void *out, int64_t out_ld, void *stream) {
  using namespace bnn;
  if (T < 0 || S < 0 || D <= 0 || k < 1 || !float_type(type)) return BNN_ERR_SHAPE;
  if (ys_ld < D || out_ld < D) return BNN_ERR_STRIDE;
  if (S > INT32_MAX || D > (1 << 28) || k > (1 << 30) || (T > 0 && k > (1 << 30) / T)) return BNN_ERR_UNSUPPORTED;
  if (T == 0) return BNN_OK;
  if ((S > 0 && !ys) || !places || !out) return BNN_ERR_NULL;
  if (!aligned16(ys) || !aligned4(places) || !aligned4(weights) || !aligned16(out)) return BNN_ERR_ALIGN;
  const int pieces = D > 512 && T * ((D - 1) / 512 + 1) > 16384 ? 2 : 1;  // more of them only where there are waves enough
  const CombineParams p = {ys, out, ys_ld, out_ld, places, weights, T, S, (D - 1) / (512 * pieces) + 1, (int)k, (int)D};
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_EXPERT_COMBINE, s);
  with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    const dim3 grid = wide_grid((T * p.chunks - 1) / 4 + 1);
    switch (row_edge(D)) {
      case EDGE_WHOLE: (pieces == 2 ? expert_combine_kernel<E, EDGE_WHOLE, 2> : expert_combine_kernel<E, EDGE_WHOLE, 1>)<<<grid, 256, 0, s>>>(p); break;
      case EDGE_RAGGED: (pieces == 2 ? expert_combine_kernel<E, EDGE_RAGGED, 2> : expert_combine_kernel<E, EDGE_RAGGED, 1>)<<<grid, 256, 0, s>>>(p); break;
      default: expert_combine_kernel<E, EDGE_SMALL, 1><<<grid, 256, 0, s>>>(p);
    }
  });
  return launch_status();
}

extern "C" bnn_status bnn_expert_combine_backward(const void *ys, int type, int64_t S, int64_t ys_ld, const int32_t *rows,
                                                  const int32_t *places, const float *weights, const void *dout, int64_t dout_ld,
                                                  int64_t T, int64_t k, int64_t D, void *dys, int64_t dys_ld, float *dweights,
                                                  void *stream) {
  using namespace bnn;
  if (T < 0 || S < 0 || D <= 0 || k < 1 || !float_type(type)) return BNN_ERR_SHAPE;
  if (dout_ld < D || (dys && dys_ld < D) || (dweights && ys_ld < D)) return BNN_ERR_STRIDE;
  if (S > INT32_MAX || D > 32768 || k > (1 << 30) || (T > 0 && k > (1 << 30) / T)) return BNN_ERR_UNSUPPORTED;
  if (!dys && !dweights) return BNN_ERR_NULL;
  if (T == 0 && (S == 0 || !dys)) return BNN_OK;
  if ((T > 0 && (!places || !dout)) || (dys && S > 0 && !rows) || (dweights && S > 0 && !ys)) return BNN_ERR_NULL;
  if (!aligned16(ys) || !aligned4(rows) || !aligned4(places) || !aligned4(weights) || !aligned16(dout) || !aligned16(dys) || !aligned4(dweights))
    return BNN_ERR_ALIGN;
  const CombineBackwardParams p = {ys, dout, dys, ys_ld, dout_ld, dys_ld, rows, places, weights, dweights, T, S, (int)k, (int)D};
  const int64_t clearing = dys ? (S + 63) / 64 : 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_EXPERT_COMBINE_BACKWARD, s);
  with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    const auto run = [&](auto whole, auto ragged, int block, int teams) {
      (row_edge(D) == EDGE_WHOLE ? whole : ragged)<<<wide_grid((T + teams - 1) / teams + clearing), block, 0, s>>>(p);
    };
#define BNN_FORMS(...) combine_backward_kernel<E, __VA_ARGS__, EDGE_WHOLE>, combine_backward_kernel<E, __VA_ARGS__, EDGE_RAGGED>
    if (D < 8) combine_backward_kernel<E, false, 256, 1, EDGE_SMALL><<<wide_grid((T + 3) / 4 + clearing), 256, 0, s>>>(p);
    else if (D <= 512) run(BNN_FORMS(false, 256, 1), 256, 4);
    else if (D <= 8192) run(BNN_FORMS(true, 1024, 1), row_threads(D, 1), 1);
    else run(BNN_FORMS(true, 1024, 4), row_threads(D, 4), 1);
#undef BNN_FORMS
  });
  return launch_status();
}
