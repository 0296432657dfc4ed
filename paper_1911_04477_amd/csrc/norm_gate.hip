// The norms after a block and before the next one, with the block's gate and residual scale between them
// (bnn_norm_gate), and their backward pass.
#include <algorithm>
#include <cmath>

#include "rows.h"

namespace bnn {

struct NormOut {
  void *r, *n;
  int64_t r_ld, n_ld, q_ld;
  int8_t *q;
  float *q_scale;
};

struct NormGrad {
  const void *dn, *dr_out;
  int64_t dn_ld, dr_out_ld;
  void *dr, *db, *dgate;
  int64_t dr_ld, db_ld, dgate_ld;
  float *part;       // [6][workers][D]: w_pre, bias_pre, w_post, bias_post, res_scale, gate
  int want;          // bit k: sum k is wanted
  int workers, per;  // teams, rows a team takes at most
  int segments;      // teams that share a group of rows with one gate; 0: a team has whole groups
};

__device__ __forceinline__ void fill8(float (&v)[8], float x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = x;
}
// A vector of D or a matrix row, `missing` where there is none: requested, and taken once it is needed.
template <class E, int EDGE>
__device__ __forceinline__ void request8(Piece8<E> &w, const E *row, const Place8<EDGE> &at, int D, float missing) {
  if (row) w.load(row, at, D);
  else w.fill(missing);
}
template <class E, int EDGE>
__device__ __forceinline__ void take8(float (&v)[8], Piece8<E> &w, const Place8<EDGE> &at) {
  if (at.shift) w.settle(at);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)w.v[j];
}

__device__ __forceinline__ void zero_past(float (&v)[8], int c, int D) {
  if (c + 8 > D)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i >= D) v[i] = 0.0f;
}

// v: values before the norm, then normed (before weight and bias).  Returns the factor.  Centred values first, then the
// mean of their squares: no difference of two large sums.  lds: two reductions' worth.  T: threads of the team.
template <bool BLOCK, int NV>
__device__ __forceinline__ void centre_rows(float (&v)[NV][8], float mean, int c0, int T, int D) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] -= mean;
    zero_past(v[i], c0 + i * T * 8, D);
  }
}
template <int NV>
__device__ __forceinline__ float sum_of(const float (&v)[NV][8]) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[i][j];
  return s;
}
template <int NV>
__device__ __forceinline__ float dot_of(const float (&v)[NV][8], const float (&u)[NV][8]) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(v[i][j], u[i][j], s);
  return s;
}
template <int NV>
__device__ __forceinline__ void times(float (&v)[NV][8], float x) {
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= x;
}
__device__ __forceinline__ float row_factor(float squares, float per, float eps) { return __builtin_amdgcn_rsqf(fmaf(squares, per, eps)); }

template <bool BLOCK, bool CENTRED, int NV>
__device__ __forceinline__ void unit_rows(float (&v)[NV][8], int norm, int c0, int T, int D, float per, float eps, uint32_t *lds) {
  if (norm == BNN_NORM_NONE) return;
  if (CENTRED && norm == BNN_NORM_LAYER) centre_rows<BLOCK, NV>(v, team_sum<BLOCK>(sum_of(v), lds) * per, c0, T, D);
  times(v, row_factor(team_sum<BLOCK>(dot_of(v, v), lds + 16), per, eps));
}

// Which row of the gate; the host has cut gate_rows to at most 2^31 - 1 rows.
__device__ __forceinline__ int64_t norm_group(const bnn_norm_gate_in &p, int64_t row) { return (uint32_t)row / (uint32_t)p.gate_rows; }

// A team (a wave, or with BLOCK a workgroup) takes a row at a time, NV pieces of eight values a thread; all that a row needs
// is requested before its first sum.  CENTRED: a norm with a mean or a bias takes part.  Bound by memory (8192 x 4096 bf16
// with a gate a token 68 us, 4.9 TB/s), a few rows by the chain of request, sum, sum.
template <class E, class R, bool BLOCK, int MAXT, int NV, bool CENTRED, int EDGE>
__global__ __launch_bounds__(MAXT) void norm_gate_kernel(bnn_norm_gate_in p, NormOut o, int teams) {
  __shared__ uint32_t lds[2 * 5 * 16];
  const int T = BLOCK ? blockDim.x : 64, t = BLOCK ? threadIdx.x : threadIdx.x & 63, c0 = t * 8, D = p.D;
  const float per = 1.0f / (float)D;
  const auto place = [&](int i) { return Place8<EDGE>(c0 + i * T * 8, D); };
  constexpr int VECTORS = CENTRED ? 5 : 3;
  const float *const from[5] = {p.w_post, p.w_pre, p.res_scale, p.bias_post, p.bias_pre};
  Piece8<float> vec[VECTORS][NV];
#pragma unroll
  for (int k = 0; k < VECTORS; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i) request8(vec[k][i], from[k], place(i), D, k < 3 ? 1.0f : 0.0f);
  bool settled = false;
  int flip = 0;  // a row's reductions do not touch what the row before left for slower waves to read
  for (int64_t row = BLOCK ? blockIdx.x : blockIdx.x * 4ll + (threadIdx.x >> 6); row < p.rows; row += teams, flip ^= 1) {
    uint32_t *const mem = lds + flip * 5 * 16;
    Piece8<E> vb[NV], vg[NV];
    Piece8<R> vr[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      request8(vb[i], p.b ? static_cast<const E *>(p.b) + row * p.b_ld : nullptr, place(i), D, 0.0f);
      vr[i].load(static_cast<const R *>(p.r) + row * p.r_ld, place(i), D);
      request8(vg[i], p.gate ? static_cast<const E *>(p.gate) + norm_group(p, row) * p.gate_ld : nullptr, place(i), D, 1.0f);
    }
    if (!settled) {  // while the first row comes
      if (BLOCK) clear_words(lds);
#pragma unroll
      for (int k = 0; k < VECTORS; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (place(i).shift) vec[k][i].settle(place(i));
      settled = true;
    }
    float v[NV][8], r[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (place(i).shift) vg[i].settle(place(i));
      take8(v[i], vb[i], place(i));
      take8(r[i], vr[i], place(i));
    }
    if (p.b) {
      unit_rows<BLOCK, CENTRED, NV>(v, p.post, c0, T, D, per, p.eps, mem);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float n = CENTRED ? fmaf(v[i][j], vec[0][i].v[j], vec[VECTORS - 2][i].v[j]) : v[i][j] * vec[0][i].v[j];
          r[i][j] = fmaf(vec[2][i].v[j] * (float)vg[i].v[j], n, r[i][j]);
        }
        if (o.r) store8(static_cast<R *>(o.r) + row * o.r_ld, c0 + i * T * 8, D, r[i]);
      }
    }
    if (p.pre == BNN_NORM_NONE) continue;
    unit_rows<BLOCK, CENTRED, NV>(r, p.pre, c0, T, D, per, p.eps, mem + 32);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) r[i][j] = CENTRED ? fmaf(r[i][j], vec[1][i].v[j], vec[VECTORS - 1][i].v[j]) : r[i][j] * vec[1][i].v[j];
      if (o.n) store8(static_cast<E *>(o.n) + row * o.n_ld, c0 + i * T * 8, D, r[i]);
    }
    if (o.q) {  // values past the end of the row are 0 in every vector
      uint32_t top = 0u;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(r[i][j]));
      const RowScale s = row_scale(team_max_magnitude<BLOCK>(top, mem + 64));
#pragma unroll
      for (int i = 0; i < NV; ++i) store_q8(o.q + row * o.q_ld, c0 + i * T * 8, D, r[i], s.inv);
      if (t == 0) o.q_scale[row] = s.scale;
    }
  }
}

// Teams walk through contiguous rows and keep the sums over rows in registers; the sums of all teams meet in
// norm_gate_sums_kernel, in the same order at every call.  A row's loads are in flight while the row before is worked on,
// and its first sum is taken along with that row's last: between rms norms a row meets twice (8192 x 4096 bf16, a workgroup
// a unit: 214 us without either, 173 with the loads ahead; with all of it 125, and 5 for the sums, 4.1 TB/s).  The vectors are
// in LDS, where there is room.  Values a thread: 8, since with 16 the sums and two rows no longer fit the registers (142 us).  CENTRED: a norm
// with a mean, a bias or the gradient of a bias takes part.
template <class E, class R, bool BLOCK, int MAXT, int NV, bool CENTRED, int EDGE>
__global__ __launch_bounds__(MAXT, NV > 1 || CENTRED ? 2 : 3) void norm_gate_backward_kernel(bnn_norm_gate_in p, NormGrad q) {
  constexpr int WIDTH = (BLOCK ? MAXT : 64) * NV * 8;
  constexpr bool NEAR = WIDTH <= 8192;
  constexpr int SUMS = 6, MEM = 8 * 16;
  __shared__ __attribute__((aligned(16))) uint32_t lds[2 * MEM];
  extern __shared__ __attribute__((aligned(16))) float near_[];  // w_post, w_pre, res_scale: as many as the teams' threads take
  const int D = p.D, width = (BLOCK ? blockDim.x : 64) * NV * 8;
  const float per = 1.0f / (float)D;
  if constexpr (NEAR) {
    const float *from[3] = {p.w_post, p.w_pre, p.res_scale};
#pragma unroll
    for (int k = 0; k < 3; ++k)
      for (int c = threadIdx.x; c < width; c += blockDim.x) near_[k * width + c] = c >= D ? 0.0f : from[k] ? from[k][c] : 1.0f;
  }
  clear_words(lds);
  const int T = BLOCK ? blockDim.x : 64, t = BLOCK ? threadIdx.x : threadIdx.x & 63, c0 = t * 8;
  const int worker = BLOCK ? blockIdx.x : blockIdx.x * 4 + (threadIdx.x >> 6);
  if (worker >= q.workers) return;  // whole waves, of workgroups without barriers from here on
  const auto place = [&](int i) { return Place8<EDGE>(c0 + i * T * 8, D); };
  const auto far = [&](float (&v)[8], const float *from, int i, float missing) {
    Piece8<float> w;
    request8(w, from, place(i), D, missing);
    take8(v, w, place(i));
  };
  const auto vector = [&](float (&v)[8], int k, int i) {
    if constexpr (NEAR) {
      const float *from = &near_[k * width + c0 + i * T * 8];
      const f32x4 lo = *reinterpret_cast<const f32x4 *>(from), hi = *reinterpret_cast<const f32x4 *>(from + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = lo[j], v[4 + j] = hi[j];
    } else {
      far(v, k == 0 ? p.w_post : k == 1 ? p.w_pre : p.res_scale, i, 1.0f);
    }
  };
  const auto bias = [&](float (&v)[8], const float *from, int i) {
    if (CENTRED) far(v, from, i, 0.0f);
    else fill8(v, 0.0f);
  };
  int row, end;
  if (q.segments) {
    const int group = worker / q.segments, part = worker % q.segments;
    const int64_t first = group * p.gate_rows + (int64_t)part * q.per;
    row = (int)min(first, p.rows);
    end = (int)min(min(first + q.per, (group + 1) * p.gate_rows), p.rows);
  } else {
    const int64_t first = (int64_t)worker * q.per;
    row = (int)min(first, p.rows);
    end = (int)min(first + q.per, p.rows);
  }
  struct Raw {
    Piece8<E> b[NV], dn[NV], g[NV];
    Piece8<R> r[NV], dro[NV];
  };
  const auto request = [&](Raw &w, int row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place8<EDGE> at = place(i);
      w.r[i].load(static_cast<const R *>(p.r) + row * p.r_ld, at, D);
      request8(w.b[i], p.b ? static_cast<const E *>(p.b) + row * p.b_ld : nullptr, at, D, 0.0f);
      request8(w.dn[i], q.dn ? static_cast<const E *>(q.dn) + row * q.dn_ld : nullptr, at, D, 0.0f);
      request8(w.dro[i], q.dr_out ? static_cast<const R *>(q.dr_out) + row * q.dr_out_ld : nullptr, at, D, 0.0f);
      request8(w.g[i], p.gate ? static_cast<const E *>(p.gate) + norm_group(p, row) * p.gate_ld : nullptr, at, D, 1.0f);
    }
  };
  float sum[SUMS][NV][8];
#pragma unroll
  for (int k = 0; k < SUMS; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i) fill8(sum[k][i], 0.0f);
  int left = (int)p.gate_rows;  // of the group with this gate
  // A row's first sum: of its squares, or (centred) of its values.
  const auto values = [&](float (&v)[NV][8], const Raw &w) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Piece8<E> x = w.b[i];
      take8(v[i], x, place(i));
    }
  };
  const bool layer_post = CENTRED && p.post == BNN_NORM_LAYER, layer_pre = CENTRED && p.pre == BNN_NORM_LAYER;
  const auto first_sum = [&](const float (&v)[NV][8]) { return layer_post ? sum_of(v) : dot_of(v, v); };
  Raw w;
  float b[NV][8], opening = 0.0f;  // of the row at hand
  if (row < end) {
    request(w, row);
    values(b, w);
    opening = team_sum<BLOCK>(first_sum(b), lds + MEM);
  }
  for (int flip = 0; row < end; ++row, flip ^= 1) {
    uint32_t *const mem = lds + flip * MEM;
    Raw ahead = w;
    if (row + 1 < end) request(ahead, row + 1);
    float r[NV][8], e[NV][8], v[8], m[8];
    // forward again: b normed, r' normed
    values(b, w);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      take8(r[i], w.r[i], place(i));
      take8(e[i], w.dn[i], place(i));
      if (place(i).shift) w.g[i].settle(place(i)), w.dro[i].settle(place(i));
    }
    float rsb = 1.0f;
    if (p.post != BNN_NORM_NONE) {
      float squares = opening;
      if (layer_post) {
        centre_rows<BLOCK, NV>(b, opening * per, c0, T, D);
        squares = team_sum<BLOCK>(dot_of(b, b), mem);
      }
      rsb = row_factor(squares, per, p.eps);
      times(b, rsb);
    }
    const auto block = [&](float (&pv)[8], int i) {  // p of this row
      float add[8];
      vector(pv, 0, i);
      bias(add, p.bias_post, i);
#pragma unroll
      for (int j = 0; j < 8; ++j) pv[j] = b[i][j] * pv[j] + add[j];
    };
    if (p.b) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        block(v, i);
        vector(m, 2, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[i][j] += m[j] * (float)w.g[i].v[j] * v[j];
        zero_past(r[i], c0 + i * T * 8, D);
      }
    }
    // gradient through the norm of r': rs (e - mean(e) - u mean(e u)), u the normed values, the first mean if centred
    if (p.pre != BNN_NORM_NONE) {
      if (layer_pre) centre_rows<BLOCK, NV>(r, team_sum<BLOCK>(sum_of(r), mem + 16) * per, c0, T, D);
      float s[3] = {dot_of(r, r), 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        vector(v, 1, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float ew = e[i][j] * v[j];
          s[1] = fmaf(ew, r[i][j], s[1]);
          if (CENTRED) s[2] += ew;
        }
      }
      team_sum<BLOCK>(s, mem + 32);
      const float rsr = row_factor(s[0], per, p.eps), along = s[1] * rsr * per, level = layer_pre ? s[2] * per : 0.0f;
      times(r, rsr);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        vector(v, 1, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum[0][i][j] = fmaf(e[i][j], r[i][j], sum[0][i][j]);
          if (CENTRED) sum[1][i][j] += e[i][j];
          e[i][j] = rsr * (e[i][j] * v[j] - level - r[i][j] * along);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) fill8(e[i], 0.0f);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {  // r from here on: the gradient of r'
#pragma unroll
      for (int j = 0; j < 8; ++j) r[i][j] = (float)w.dro[i].v[j] + e[i][j];
      zero_past(r[i], c0 + i * T * 8, D);
      store8(static_cast<R *>(q.dr) + row * q.dr_ld, c0 + i * T * 8, D, r[i]);
    }
    if (p.b) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        block(v, i);
        vector(m, 2, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float g = (float)w.g[i].v[j], along = r[i][j] * v[j], dp = r[i][j] * m[j] * g;
          sum[2][i][j] = fmaf(dp, b[i][j], sum[2][i][j]);
          if (CENTRED) sum[3][i][j] += dp;
          sum[4][i][j] = fmaf(along, g, sum[4][i][j]);
          sum[5][i][j] = fmaf(along, m[j], sum[5][i][j]);
          e[i][j] = dp;
        }
        vector(v, 0, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) e[i][j] *= v[j];
      }
      float next[NV][8];
      values(next, ahead);
      float s[3] = {dot_of(e, b), first_sum(next), CENTRED ? sum_of(e) : 0.0f};
      team_sum<BLOCK>(s, mem + 80);
      opening = s[1];
      if (p.post != BNN_NORM_NONE) {
        const float along = s[0] * per, level = layer_post ? s[2] * per : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) e[i][j] = rsb * (e[i][j] - level - b[i][j] * along);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) store8(static_cast<E *>(q.db) + row * q.db_ld, c0 + i * T * 8, D, e[i]);
      if (q.dgate && !q.segments && (--left == 0 || row + 1 == end)) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          store8(static_cast<E *>(q.dgate) + norm_group(p, row) * q.dgate_ld, c0 + i * T * 8, D, sum[5][i]);
          fill8(sum[5][i], 0.0f);
        }
        left = (int)p.gate_rows;
      }
    }
    w = ahead;
  }
#pragma unroll
  for (int k = 0; k < SUMS; ++k)
    if (q.want >> k & 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) store8(q.part + ((int64_t)k * q.workers + worker) * D, c0 + i * T * 8, D, sum[k][i]);
}

struct NormSums {
  const float *part;
  float *out[5];
  void *dgate;
  int64_t dgate_ld;
  int workers, segments, D;
};
// Sums of the teams' sums: 64 columns a workgroup, its 16 waves share the teams out.  blockIdx.y: which sum; from 5 on: the
// gate of group blockIdx.y - 5.
template <class E>
__global__ __launch_bounds__(1024) void norm_gate_sums_kernel(NormSums q) {
  __shared__ float lds[16][64];
  const int which = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  if (which < 5 && !q.out[which]) return;
  const int first = which < 5 ? 0 : (which - 5) * q.segments, last = which < 5 ? q.workers : first + q.segments;
  const float *part = q.part + (int64_t)min(which, 5) * q.workers * q.D;
  float sum = 0.0f;
  if (c < q.D) {
    int w = first + wave;
    for (; w + 48 < last; w += 64) {  // four in flight
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = part[(int64_t)(w + 16 * i) * q.D + c];
      sum += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; w < last; w += 16) sum += part[(int64_t)w * q.D + c];
  }
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave || c >= q.D) return;
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += lds[w][lane];
  if (which < 5) q.out[which][c] = sum;
  else static_cast<E *>(q.dgate)[(which - 5) * q.dgate_ld + c] = (E)sum;
}

constexpr int NORM_MAX_D = 16384;

struct NormPlan {
  int workers, per, segments;
};
// As many teams as run at once on 256 units, about (the workspace's size follows from it, and is asked for without a device); each takes contiguous rows, of one group where a gate is shared by more rows than
// that, else of whole groups.  at_once: waves of the kernel that a compute unit has registers for.
constexpr int NORM_WAVES = 12, NORM_WAVES_CENTRED = 8;
inline NormPlan norm_plan(int64_t rows, int D, int64_t gate_rows, int at_once) {
  const int64_t waves = (D + 511) / 512, room = 256 * std::max<int64_t>(1, at_once / waves);
  int64_t per = (rows - 1) / room + 1;
  if (gate_rows > rows) gate_rows = rows;
  if (gate_rows > per) {
    const int64_t segments = (gate_rows - 1) / per + 1, groups = (rows - 1) / gate_rows + 1;
    return {(int)(segments * groups), (int)((gate_rows - 1) / segments + 1), (int)segments};
  }
  if (gate_rows > 0) per = ((per - 1) / gate_rows + 1) * gate_rows;
  return {(int)((rows - 1) / per + 1), (int)per, 0};
}

// f with the element types as tags.
template <class F>
void with_norm(const bnn_norm_gate_in &p, const F &f) {
  if (p.type == BNN_F32) f(0.0f, 0.0f);
  else if (p.type == BNN_BF16 && p.r_type == BNN_F32) f((__bf16)0.0f, 0.0f);
  else if (p.type == BNN_BF16) f((__bf16)0.0f, (__bf16)0.0f);
  else if (p.r_type == BNN_F32) f((_Float16)0.0f, 0.0f);
  else f((_Float16)0.0f, (_Float16)0.0f);
}

inline bool norm_known(int n) { return n >= BNN_NORM_NONE && n <= BNN_NORM_LAYER; }

// No group is longer than the rows there are.
inline bnn_norm_gate_in cut_groups(bnn_norm_gate_in p) {
  p.gate_rows = p.gate ? std::min(p.gate_rows, p.rows) : 1;
  return p;
}

inline bool has_means(const bnn_norm_gate_in &p) {
  return p.post == BNN_NORM_LAYER || p.pre == BNN_NORM_LAYER || p.bias_post || p.bias_pre;
}

bnn_status check_norm(const bnn_norm_gate_in *p) {
  if (!p) return BNN_ERR_NULL;
  if (p->rows < 0 || p->D <= 0 || !float_type(p->type) || !float_type(p->r_type) || !norm_known(p->post) || !norm_known(p->pre) ||
      !(p->eps >= 0.0f) || !std::isfinite(p->eps))
    return BNN_ERR_SHAPE;
  if (p->gate && p->gate_rows < 1) return BNN_ERR_SHAPE;
  if (p->rows > 0 && !p->b && (p->post != BNN_NORM_NONE || p->gate || p->res_scale)) return BNN_ERR_NULL;  // of nothing
  if ((p->post == BNN_NORM_NONE && (p->w_post || p->bias_post)) || (p->pre == BNN_NORM_NONE && (p->w_pre || p->bias_pre)))
    return BNN_ERR_SHAPE;
  if (p->r_ld < p->D || (p->b && p->b_ld < p->D) || (p->gate && p->gate_ld < p->D)) return BNN_ERR_STRIDE;
  if ((p->r_type != p->type && p->r_type != BNN_F32) || p->D > NORM_MAX_D || p->rows > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  if (!aligned16(p->b) || !aligned16(p->r) || !aligned16(p->gate) || !aligned16(p->res_scale) || !aligned16(p->w_post) ||
      !aligned16(p->bias_post) || !aligned16(p->w_pre) || !aligned16(p->bias_pre))
    return BNN_ERR_ALIGN;
  return BNN_OK;
}

}  // namespace bnn

extern "C" bnn_status bnn_norm_gate(const bnn_norm_gate_in *in, void *r_out, int64_t r_out_ld, void *n_out, int64_t n_ld, int8_t *q_out,
                                    int64_t q_ld, float *q_scale, void *stream) {
  using namespace bnn;
  if (bnn_status st = check_norm(in)) return st;
  const bnn_norm_gate_in &p = *in;
  if (p.pre == BNN_NORM_NONE && (n_out || q_out)) return BNN_ERR_SHAPE;
  if ((r_out && r_out_ld < p.D) || (n_out && n_ld < p.D) || (q_out && q_ld < p.D)) return BNN_ERR_STRIDE;
  if (p.rows == 0) return BNN_OK;
  if (!p.r || (p.b && !r_out) || (!p.b && r_out) || (p.pre != BNN_NORM_NONE && !n_out && !q_out) || (!q_out != !q_scale))
    return BNN_ERR_NULL;
  if (!aligned16(r_out) || !aligned16(n_out) || !aligned16(q_out) || !aligned16(q_scale)) return BNN_ERR_ALIGN;
  if (!p.b && p.pre == BNN_NORM_NONE) return BNN_OK;  // nothing to write
  const NormOut o = {r_out, n_out, r_out_ld, n_ld, q_ld, q_out, q_scale};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bnn_norm_gate_in in_groups = cut_groups(p);
  const bool centred = has_means(p);
  const RowEdge edge = row_edge(p.D);
  ProfScope ps(KID_NORM_GATE, s);
  with_norm(p, [&](auto e, auto r) {
    using E = decltype(e);
    using R = decltype(r);
    const auto run = [&](auto plain, auto with_means, auto ragged, int block, int teams) {  // as many workgroups as run at once, at most
      const uint32_t grid = (uint32_t)std::min<int64_t>((p.rows - 1) / teams + 1, 256 * (2048 / block));
      (edge != EDGE_WHOLE ? ragged : centred ? with_means : plain)<<<grid, block, 0, s>>>(in_groups, o, (int)grid * teams);
    };
// rows of a multiple of eight values without and with means, and any others
#define BNN_FORMS(kernel, ...) \
  kernel<E, R, __VA_ARGS__, false, EDGE_WHOLE>, kernel<E, R, __VA_ARGS__, true, EDGE_WHOLE>, kernel<E, R, __VA_ARGS__, true, EDGE_RAGGED>
#define BNN_SMALL(kernel) kernel<E, R, false, 256, 1, true, EDGE_SMALL>
    if (edge == EDGE_SMALL) run(BNN_SMALL(norm_gate_kernel), BNN_SMALL(norm_gate_kernel), BNN_SMALL(norm_gate_kernel), 256, 4);
    else if (p.D <= 512) run(BNN_FORMS(norm_gate_kernel, false, 256, 1), 256, 4);
    else if (p.D <= 4096) run(BNN_FORMS(norm_gate_kernel, true, 512, 1), row_threads(p.D, 1), 1);
    else if (p.D <= 8192) run(BNN_FORMS(norm_gate_kernel, true, 1024, 1), row_threads(p.D, 1), 1);
    else run(BNN_FORMS(norm_gate_kernel, true, 1024, 2), row_threads(p.D, 2), 1);
  });
  return launch_status();
}

extern "C" size_t bnn_norm_gate_backward_workspace_bytes(int64_t rows, int D, int64_t gate_rows) {
  using namespace bnn;
  if (rows <= 0 || D <= 0 || D > NORM_MAX_D || rows > INT32_MAX || gate_rows < 0) return 0;
  return sizeof(float) * 6 * (size_t)norm_plan(rows, D, gate_rows, NORM_WAVES).workers * (size_t)D;  // no other plan has more
}

extern "C" bnn_status bnn_norm_gate_backward(const bnn_norm_gate_in *in, const void *dn, int64_t dn_ld, const void *dr_out,
                                             int64_t dr_out_ld, void *dr, int64_t dr_ld, void *db, int64_t db_ld, void *dgate,
                                             int64_t dgate_ld, float *dres_scale, float *dw_post, float *dbias_post, float *dw_pre,
                                             float *dbias_pre, void *workspace, size_t workspace_bytes, void *stream) {
  using namespace bnn;
  if (bnn_status st = check_norm(in)) return st;
  const bnn_norm_gate_in &p = *in;
  if (p.pre == BNN_NORM_NONE && (dn || dw_pre || dbias_pre)) return BNN_ERR_SHAPE;
  if (p.rows > 0 && ((!p.b && (db || dres_scale || dw_post || dbias_post)) || (!p.gate && dgate))) return BNN_ERR_SHAPE;
  if ((dn && dn_ld < p.D) || (dr_out && dr_out_ld < p.D) || (dr && dr_ld < p.D) || (db && db_ld < p.D) || (dgate && dgate_ld < p.D))
    return BNN_ERR_STRIDE;
  if (!aligned16(dn) || !aligned16(dr_out) || !aligned16(dr) || !aligned16(db) || !aligned16(dgate) || !aligned16(dres_scale) ||
      !aligned16(dw_post) || !aligned16(dbias_post) || !aligned16(dw_pre) || !aligned16(dbias_pre) || !aligned16(workspace))
    return BNN_ERR_ALIGN;
  NormSums sums = {};
  sums.D = p.D;
  sums.out[0] = dw_pre, sums.out[1] = dbias_pre, sums.out[2] = dw_post, sums.out[3] = dbias_post, sums.out[4] = dres_scale;
  NormGrad q = {};
  for (int k = 0; k < 5; ++k) q.want |= (sums.out[k] ? 1 : 0) << k;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.rows > 0) {
    if (!p.r || !dr || (p.b && !db)) return BNN_ERR_NULL;
    const bool centred = has_means(p) || dbias_post || dbias_pre;  // the gradient of a bias is one where the bias is absent, too
    const RowEdge edge = row_edge(p.D);
    const NormPlan plan = norm_plan(p.rows, p.D, p.gate ? p.gate_rows : 0, centred || edge != EDGE_WHOLE ? NORM_WAVES_CENTRED : NORM_WAVES);
    q.dn = dn, q.dr_out = dr_out, q.dn_ld = dn_ld, q.dr_out_ld = dr_out_ld;
    q.dr = dr, q.db = db, q.dgate = dgate, q.dr_ld = dr_ld, q.db_ld = db_ld, q.dgate_ld = dgate_ld;
    q.workers = plan.workers, q.per = plan.per, q.segments = plan.segments;
    if (dgate && plan.segments) q.want |= 1 << 5;
    if (q.want) {
      if (!workspace) return BNN_ERR_NULL;
      if (workspace_bytes < bnn_norm_gate_backward_workspace_bytes(p.rows, p.D, p.gate ? p.gate_rows : 0)) return BNN_ERR_WORKSPACE;
    }
    q.part = static_cast<float *>(workspace);
    const bnn_norm_gate_in in_groups = cut_groups(p);
    ProfScope ps(KID_NORM_GATE_BACKWARD, s);
    with_norm(p, [&](auto e, auto r) {
      using E = decltype(e);
      using R = decltype(r);
      const auto run = [&](auto plain, auto with_means, auto ragged, int block, int teams) {
        const size_t near_bytes = p.D <= 8192 ? 3 * sizeof(float) * (size_t)(p.D <= 512 ? 512 : p.D <= 4096 ? row_threads(p.D, 1) * 8 : row_threads(p.D, 2) * 16) : 0;
        (edge != EDGE_WHOLE ? ragged : centred ? with_means : plain)<<<(uint32_t)((plan.workers - 1) / teams + 1), block, near_bytes, s>>>(in_groups, q);
      };
      if (edge == EDGE_SMALL)
        run(BNN_SMALL(norm_gate_backward_kernel), BNN_SMALL(norm_gate_backward_kernel), BNN_SMALL(norm_gate_backward_kernel), 256, 4);
      else if (p.D <= 512) run(BNN_FORMS(norm_gate_backward_kernel, false, 256, 1), 256, 4);
      else if (p.D <= 4096) run(BNN_FORMS(norm_gate_backward_kernel, true, 512, 1), row_threads(p.D, 1), 1);
      else if (p.D <= 8192) run(BNN_FORMS(norm_gate_backward_kernel, true, 512, 2), row_threads(p.D, 2), 1);
      else run(BNN_FORMS(norm_gate_backward_kernel, true, 1024, 2), row_threads(p.D, 2), 1);
#undef BNN_FORMS
#undef BNN_SMALL
    });
    if (bnn_status st = launch_status()) return st;
  } else if (!q.want) {
    return BNN_OK;
  }
  if (q.want) {
    sums.part = q.part, sums.workers = q.workers, sums.segments = q.segments, sums.dgate = dgate, sums.dgate_ld = dgate_ld;
    const uint32_t groups = q.want >> 5 & 1 ? (uint32_t)(q.workers / q.segments) : 0u;
    ProfScope ps(KID_NORM_GATE_SUMS, s);
    with_float(p.type, [&](auto tag) {
      norm_gate_sums_kernel<typename decltype(tag)::type><<<dim3((uint32_t)(p.D - 1) / 64 + 1, 5 + groups), 1024, 0, s>>>(sums);
    });
  }
  return launch_status();
}
