// Floating-point values as e4m3 with a scale for each block of 128 (bnn_quant_blocks_f8, bnn_quant_columns_f8,
// bnn_quant_weight_f8): activations in blocks along a row, or along a column for a weight's gradient; weights in blocks of
// 128 x 128, both as they lie and transposed.
#include "f8.h"

namespace bnn {

// Which rows of x are taken: all T, or for each of S positions the token of a slot (bnn_expert_sort).
struct F8Source {
  const void *x;
  int64_t ld, T;
  const int32_t *rows;
  FastDiv k;
  int64_t slots;  // T * k
  int64_t S;
  // x's row at position p: -1 zeros, -2 left alone
  __device__ __forceinline__ int64_t row(int64_t p) const {
    if (!rows) return p;
    const int r = rows[p];
    return r >= 0 && r < slots ? (int64_t)fdiv((uint32_t)r, k) : r == -1 ? -1 : -2;
  }
};

struct QuantBlocksParams {
  F8Source src;
  int K, blocks;
  FastDiv by;  // blocks
  uint8_t *q, *scale;
  int64_t q_ld, scale_ld, total;
};

// Sixteen lanes a block, eight values each: the maximum is four steps among them, without LDS.  Bound by memory (8192 x 8192 bf16, 134 MB in, 68
// out, 38 to 41 us, 5.1 TB/s; four blocks a lane are no faster).
template <class E, int EDGE>
__global__ __launch_bounds__(256) void quant_blocks_kernel(QuantBlocksParams p) {
  const int64_t id = wide_block() * 16 + (threadIdx.x >> 4);
  if (id >= p.total) return;  // whole rows of lanes
  int64_t at;
  int block;
  if (p.total < (1ll << 31)) {
    const uint32_t row = fdiv((uint32_t)id, p.by);
    at = row, block = (int)((uint32_t)id - row * (uint32_t)p.blocks);
  } else {
    at = id / p.blocks, block = (int)(id - at * p.blocks);
  }
  const int64_t row = p.src.row(at);
  if (row < -1) return;
  const int c = block * F8_BLOCK + (threadIdx.x & 15) * 8;
  float v[8] = {};
  if (row >= 0) {
    const Place8<EDGE> place(c, p.K);
    Piece8<E> x;
    x.load(static_cast<const E *>(p.src.x) + row * p.src.ld, place, p.K);
    if (place.shift) x.settle(place);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)x.v[i];
  }
  f8_store_block(v, p.q + at * p.q_ld, p.scale + at * p.scale_ld, c);
}

struct QuantColumnsParams {
  F8Source src;
  int D, blocks;  // columns of x; blocks of positions
  uint8_t *q, *scale;
  int64_t q_ld, scale_ld;
};

// 128 positions by 64 columns a workgroup: a thread reads eight columns of four consecutive positions, the columns' maxima meet
// in LDS, and the bytes are turned there, so that a column's block leaves as one line of 128 bytes (8192 x 4096 bf16 21 to 24 us, 4.3 TB/s).
constexpr int QC_PITCH = F8_BLOCK + 16;
template <class E, int EDGE>
__global__ __launch_bounds__(256) void quant_columns_kernel(QuantColumnsParams p) {
  __shared__ uint32_t tops[4][64];
  __shared__ __attribute__((aligned(16))) uint8_t turned[64 * QC_PITCH];
  const int t = threadIdx.x, group = t & 7, four = t >> 3;
  const int64_t s0 = (int64_t)blockIdx.y * F8_BLOCK;
  const int c = blockIdx.x * 64 + group * 8;
  Piece8<E> x[4];
  const Place8<EDGE> place(c, p.D);
  int64_t row[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t s = s0 + four * 4 + i;
    row[i] = s < p.src.S ? p.src.row(s) : -1;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i].load(static_cast<const E *>(p.src.x) + max(row[i], (int64_t)0) * p.src.ld, place, p.D);
  uint32_t top[8] = {};
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (place.shift) x[i].settle(place);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[i][j] = row[i] >= 0 ? (float)x[i].v[j] : 0.0f;
      top[j] = max(top[j], f8_magnitude(v[i][j]));
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int d = 8; d < 64; d *= 2) top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], d));
  }
  if ((t & 63) < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) tops[t >> 6][group * 8 + j] = top[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int col = group * 8 + j;
    const uint32_t byte = f8_scale_byte(max(max(tops[0][col], tops[1][col]), max(tops[2][col], tops[3][col])));
    const float inv = f8_inverse(byte);
    *reinterpret_cast<uint32_t *>(turned + col * QC_PITCH + four * 4) = f8_pack(v[0][j] * inv, v[1][j] * inv, v[2][j] * inv, v[3][j] * inv);
    if (four == 0 && blockIdx.x * 64 + col < p.D) p.scale[(int64_t)(blockIdx.x * 64 + col) * p.scale_ld + blockIdx.y] = (uint8_t)byte;
  }
  __syncthreads();
  const int col = t >> 2, part = (t & 3) * 32;
  if (blockIdx.x * 64 + col >= p.D) return;
  uint8_t *to = p.q + (int64_t)(blockIdx.x * 64 + col) * p.q_ld + s0 + part;
  const u32x4 *from = reinterpret_cast<const u32x4 *>(turned + col * QC_PITCH + part);
  reinterpret_cast<u32x4 *>(to)[0] = from[0];
  reinterpret_cast<u32x4 *>(to)[1] = from[1];
}

struct QuantWeightParams {
  const void *w;
  int64_t ld, es;
  int N, K;
  bnn_f8_weight out, turned;
};

// A block of 128 x 128 a workgroup: 64 values a thread in registers between the maximum and the rounding, so that both forms come from one
// reading (4096 x 4096 bf16, 34 MB in, 34 out, 17 us, 3.9 TB/s).
template <class E, int EDGE>
__global__ __launch_bounds__(256) void quant_weight_kernel(QuantWeightParams p) {
  __shared__ uint32_t tops[4];
  __shared__ __attribute__((aligned(16))) uint8_t turned[F8_BLOCK * QC_PITCH];
  const int t = threadIdx.x, group = t & 15, four = t >> 4;  // eight columns; rows 4 * four + i and 64 further on
  const int n0 = blockIdx.y * F8_BLOCK, c = blockIdx.x * F8_BLOCK + group * 8;
  const int64_t e = blockIdx.z;
  const E *w = static_cast<const E *>(p.w) + e * p.es;
  const Place8<EDGE> place(c, p.K);
  Piece8<E> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i].load(w + (int64_t)min(n0 + four * 4 + (i >> 2) * 64 + (i & 3), p.N - 1) * p.ld, place, p.K);
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (place.shift) x[i].settle(place);
    if (n0 + four * 4 + (i >> 2) * 64 + (i & 3) >= p.N) x[i].fill(0.0f);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, f8_magnitude((float)x[i].v[j]));
  }
  top = (uint32_t)wave_reduce(top, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  if ((t & 63) == 0) tops[t >> 6] = top;
  __syncthreads();
  const uint32_t byte = f8_scale_byte(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  const float inv = f8_inverse(byte);
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if (p.out.q) {
    uint8_t *q = static_cast<uint8_t *>(p.out.q) + e * p.out.expert_ld;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int n = n0 + four * 4 + (i >> 2) * 64 + (i & 3);
      const auto &v = x[i].v;
      if (n < p.N)
        *reinterpret_cast<u32x2 *>(q + (int64_t)n * p.out.ld + c) =
            u32x2{f8_pack((float)v[0] * inv, (float)v[1] * inv, (float)v[2] * inv, (float)v[3] * inv),
                  f8_pack((float)v[4] * inv, (float)v[5] * inv, (float)v[6] * inv, (float)v[7] * inv)};
    }
    if (t == 0) p.out.scale[e * p.out.scale_expert_ld + blockIdx.y * p.out.scale_ld + blockIdx.x] = (uint8_t)byte;
  }
  if (p.turned.q) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<uint32_t *>(turned + (group * 8 + j) * QC_PITCH + h * 64 + four * 4) =
            f8_pack((float)x[h * 4].v[j] * inv, (float)x[h * 4 + 1].v[j] * inv, (float)x[h * 4 + 2].v[j] * inv, (float)x[h * 4 + 3].v[j] * inv);
    __syncthreads();
    uint8_t *q = static_cast<uint8_t *>(p.turned.q) + e * p.turned.expert_ld;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = i * 32 + (t >> 3), part = (t & 7) * 16, k = blockIdx.x * F8_BLOCK + col;
      if (k < p.K)
        *reinterpret_cast<u32x4 *>(q + (int64_t)k * p.turned.ld + n0 + part) = *reinterpret_cast<const u32x4 *>(turned + col * QC_PITCH + part);
    }
    if (t == 0) p.turned.scale[e * p.turned.scale_expert_ld + blockIdx.x * p.turned.scale_ld + blockIdx.y] = (uint8_t)byte;
  }
}

F8Source f8_source(const void *x, int64_t x_ld, int64_t T, const int32_t *rows, int64_t k, int64_t S) {
  return {x, x_ld, T, rows, FastDiv(rows ? (uint32_t)k : 1u), rows ? T * k : 0, S};
}

template <class F>
void f8_edges(int64_t K, const F &f) {
  switch (row_edge(K)) {
    case EDGE_WHOLE: return f(std::integral_constant<int, EDGE_WHOLE>());
    case EDGE_RAGGED: return f(std::integral_constant<int, EDGE_RAGGED>());
    default: return f(std::integral_constant<int, EDGE_SMALL>());
  }
}

bool f8_sizes_fit(int64_t T, int64_t k, int64_t S, int64_t K, const int32_t *rows) {
  return T <= INT32_MAX && S <= INT32_MAX && K <= (1 << 28) && (!rows || k <= INT32_MAX / (T > 0 ? T : 1));
}

}  // namespace bnn

extern "C" int64_t bnn_f8_row_bytes(int64_t K) { return K <= 0 ? 0 : bnn::f8_row_bytes(K); }
extern "C" int64_t bnn_f8_scale_bytes(int64_t K) { return K <= 0 ? 0 : bnn::f8_scale_bytes(K); }

extern "C" bnn_status bnn_quant_blocks_f8(const void *x, int type, int64_t T, int64_t x_ld, const int32_t *rows, int64_t k,
                                          int64_t S, int64_t K, uint8_t *q, int64_t q_ld, uint8_t *scale, int64_t scale_ld,
                                          void *stream) {
  using namespace bnn;
  if (T < 0 || S < 0 || K <= 0 || !float_type(type) || (rows ? k < 1 : S != T)) return BNN_ERR_SHAPE;
  if (x_ld < K) return BNN_ERR_STRIDE;
  if (!f8_sizes_fit(T, k, S, K, rows)) return BNN_ERR_UNSUPPORTED;
  if (S == 0) return BNN_OK;
  const bnn_status st = f8_check(q, q_ld, scale, scale_ld, K, false);
  if (st != BNN_OK) return st;
  if (!x && T > 0) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned4(rows)) return BNN_ERR_ALIGN;
  QuantBlocksParams p = {};
  p.src = f8_source(x, x_ld, T, rows, k, S);
  p.K = (int)K, p.blocks = (int)f8_blocks(K), p.by = FastDiv((uint32_t)p.blocks);
  p.q = q, p.scale = scale, p.q_ld = q_ld, p.scale_ld = scale_ld, p.total = S * p.blocks;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_QUANT_F8, s);
  with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    f8_edges(K, [&](auto edge) { quant_blocks_kernel<E, decltype(edge)::value><<<wide_grid((p.total - 1) / 16 + 1), 256, 0, s>>>(p); });
  });
  return launch_status();
}

extern "C" bnn_status bnn_quant_columns_f8(const void *x, int type, int64_t T, int64_t x_ld, const int32_t *rows, int64_t k,
                                           int64_t S, int64_t D, uint8_t *q, int64_t q_ld, uint8_t *scale, int64_t scale_ld,
                                           void *stream) {
  using namespace bnn;
  if (T < 0 || S < 0 || D <= 0 || !float_type(type) || (rows ? k < 1 : S != T)) return BNN_ERR_SHAPE;
  if (x_ld < D) return BNN_ERR_STRIDE;
  if (!f8_sizes_fit(T, k, S, D, rows) || S > F8_MOST_K) return BNN_ERR_UNSUPPORTED;
  if (S == 0) return BNN_OK;
  const bnn_status st = f8_check(q, q_ld, scale, scale_ld, S, false);
  if (st != BNN_OK) return st;
  if (!x && T > 0) return BNN_ERR_NULL;
  if (!aligned16(x) || !aligned4(rows)) return BNN_ERR_ALIGN;
  if (T == 0) return BNN_ERR_SHAPE;  // S positions of no rows
  QuantColumnsParams p = {};
  p.src = f8_source(x, x_ld, T, rows, k, S);
  p.D = (int)D, p.blocks = (int)f8_blocks(S), p.q = q, p.scale = scale, p.q_ld = q_ld, p.scale_ld = scale_ld;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_QUANT_F8_COLUMNS, s);
  with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    f8_edges(D, [&](auto edge) {
      quant_columns_kernel<E, decltype(edge)::value><<<dim3((uint32_t)((D - 1) / 64 + 1), (uint32_t)p.blocks), 256, 0, s>>>(p);
    });
  });
  return launch_status();
}

extern "C" bnn_status bnn_quant_weight_f8(const void *w, int type, int64_t experts, int64_t expert_ld, int64_t N, int64_t K,
                                          int64_t w_ld, const bnn_f8_weight *out, const bnn_f8_weight *turned, void *stream) {
  using namespace bnn;
  if (experts < 0 || N <= 0 || K <= 0 || !float_type(type)) return BNN_ERR_SHAPE;
  if (w_ld < K || (experts > 1 && expert_ld < 0)) return BNN_ERR_STRIDE;
  if (experts > 65535 || N > (1 << 22) || K > (1 << 22) || (out && K > F8_MOST_K) || (turned && N > F8_MOST_K)) return BNN_ERR_UNSUPPORTED;
  if (experts == 0) return BNN_OK;
  if (!w || (!out && !turned)) return BNN_ERR_NULL;
  QuantWeightParams p = {w, w_ld, expert_ld, (int)N, (int)K, {}, {}};
  for (int i = 0; i < 2; ++i) {
    const bnn_f8_weight *o = i ? turned : out;
    if (!o) continue;
    const int64_t rows = i ? K : N, cols = i ? N : K;
    const bnn_status st = f8_check(o->q, o->ld, o->scale, o->scale_ld, cols, false);
    if (st != BNN_OK) return st;
    if (experts > 1 && (o->expert_ld / rows < o->ld || o->expert_ld % 16 || o->scale_expert_ld / f8_blocks(rows) < o->scale_ld || o->scale_expert_ld % 4))
      return BNN_ERR_STRIDE;
    (i ? p.turned : p.out) = *o;
  }
  if (!aligned16(w)) return BNN_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(KID_QUANT_F8_WEIGHT, s);
  with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    f8_edges(K, [&](auto edge) {
      quant_weight_kernel<E, decltype(edge)::value><<<dim3((uint32_t)f8_blocks(K), (uint32_t)f8_blocks(N), (uint32_t)experts), 256, 0, s>>>(p);
    });
  });
  return launch_status();
}
