// The activation of gated projections that lie side by side, gu = [g | u] as one product gives them: h = act(g) * u in floating
// point or as e4m3 rows with block scales, and its gradient (bnn_gated_act, bnn_gated_act_f8, bnn_gated_act_backward).
// Bound by memory.
#include "activation.h"
#include "f8.h"

namespace bnn {

struct GatedActParams {
  const void *gu, *dh;
  void *out;       // h, or dgu
  uint8_t *q, *scale;
  int64_t gu_ld, dh_ld, out_ld, q_ld, scale_ld;
  const int32_t *live;  // rows from *live on are left alone
  int64_t total;   // pieces of all rows
  int F, pieces, act;
  FastDiv by;
};

enum : int { GATE_FLOAT, GATE_F8, GATE_BACKWARD };

// Eight columns a thread.  Bound by memory (16384 x 4096 bf16: 403 MB 72 us, 5.6 TB/s; gradient 671 MB 114 us, 5.9).
template <class E, int EDGE, int FORM, int ACT>
__global__ __launch_bounds__(256) void gated_act_kernel(GatedActParams p) {
  const int64_t id = wide_block() * 256 + threadIdx.x;
  if (id >= p.total) return;  // e4m3: whole blocks of 16 lanes
  int64_t row;
  int piece;
  if (p.total < (1ll << 31)) {
    const uint32_t r = fdiv((uint32_t)id, p.by);
    row = r, piece = (int)((uint32_t)id - r * (uint32_t)p.pieces);
  } else {
    row = id / p.pieces, piece = (int)(id - row * p.pieces);
  }
  if (p.live && row >= *p.live) return;
  const int c = piece * 8;
  const Place8<EDGE> at(c, p.F);
  const E *g = static_cast<const E *>(p.gu) + row * p.gu_ld;
  Piece8<E> vg, vu, vd;
  vg.load(g, at, p.F);
  vu.load(g + p.F, at, p.F);
  if constexpr (FORM == GATE_BACKWARD) vd.load(static_cast<const E *>(p.dh) + row * p.dh_ld, at, p.F);
  if (at.shift) {
    vg.settle(at), vu.settle(at);
    if constexpr (FORM == GATE_BACKWARD) vd.settle(at);
  }
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float z = (float)vg.v[i], u = (float)vu.v[i];
    float slope;
    const float y = activation<FORM == GATE_BACKWARD>(ACT, z, slope);
    if constexpr (FORM == GATE_BACKWARD) {
      const float d = (float)vd.v[i];
      a[i] = d * u * slope, b[i] = d * y;
    } else {
      a[i] = y * u;
    }
  }
  if constexpr (FORM == GATE_F8) {
    f8_store_block(a, p.q + row * p.q_ld, p.scale + row * p.scale_ld, c);
  } else {
    E *out = static_cast<E *>(p.out) + row * p.out_ld;
    store8(out, c, p.F, a);
    if constexpr (FORM == GATE_BACKWARD) store8(out + p.F, c, p.F, b);
  }
}

template <int FORM>
bnn_status run_gated_act(GatedActParams &p, int type, int64_t S, hipStream_t s) {
  p.pieces = FORM == GATE_F8 ? (int)f8_row_bytes(p.F) / 8 : (p.F + 7) / 8;
  p.by = FastDiv((uint32_t)p.pieces);
  p.total = S * p.pieces;
  ProfScope ps(FORM == GATE_BACKWARD ? KID_GATED_ACT_BACKWARD : KID_GATED_ACT, s);
  return with_float(type, [&](auto tag) {
    using E = typename decltype(tag)::type;
    return with_act(p.act, [&](auto act) {
      constexpr int ACT = decltype(act)::value;
      const dim3 grid = wide_grid((p.total - 1) / 256 + 1);
      switch (row_edge(p.F)) {
        case EDGE_WHOLE: gated_act_kernel<E, EDGE_WHOLE, FORM, ACT><<<grid, 256, 0, s>>>(p); break;
        case EDGE_RAGGED: gated_act_kernel<E, EDGE_RAGGED, FORM, ACT><<<grid, 256, 0, s>>>(p); break;
        default: gated_act_kernel<E, EDGE_SMALL, FORM, ACT><<<grid, 256, 0, s>>>(p);
      }
      return launch_status();
    });
  });
}

bnn_status check_gated_act(const void *gu, int type, int64_t S, int64_t gu_ld, int64_t F, int act) {
  if (S < 0 || F <= 0 || !float_type(type) || act < BNN_ACT_SILU || act > BNN_ACT_RELU) return BNN_ERR_SHAPE;
  if (gu_ld < 2 * F) return BNN_ERR_STRIDE;
  if (F > (1 << 28) || S > INT32_MAX) return BNN_ERR_UNSUPPORTED;
  if (S == 0) return BNN_OK;
  if (!gu) return BNN_ERR_NULL;
  return aligned16(gu) ? BNN_OK : BNN_ERR_ALIGN;
}

}  // namespace bnn

extern "C" bnn_status bnn_gated_act(const void *gu, int type, int64_t S, int64_t gu_ld, int64_t F, int act, const int32_t *live, void *h,
                                    int64_t h_ld, void *stream) {
  using namespace bnn;
  const bnn_status st = check_gated_act(gu, type, S, gu_ld, F, act);
  if (st != BNN_OK) return st;
  if (h_ld < F) return BNN_ERR_STRIDE;
  if (S == 0) return BNN_OK;
  if (!h) return BNN_ERR_NULL;
  if (!aligned16(h) || !aligned4(live)) return BNN_ERR_ALIGN;
  GatedActParams p = {};
  p.gu = gu, p.gu_ld = gu_ld, p.F = (int)F, p.act = act, p.live = live, p.out = h, p.out_ld = h_ld;
  return run_gated_act<GATE_FLOAT>(p, type, S, static_cast<hipStream_t>(stream));
}

extern "C" bnn_status bnn_gated_act_f8(const void *gu, int type, int64_t S, int64_t gu_ld, int64_t F, int act, const int32_t *live,
                                       uint8_t *q, int64_t q_ld, uint8_t *scale, int64_t scale_ld, void *stream) {
  using namespace bnn;
  bnn_status st = check_gated_act(gu, type, S, gu_ld, F, act);
  if (st != BNN_OK) return st;
  if (S == 0) return BNN_OK;
  st = f8_check(q, q_ld, scale, scale_ld, F, false);
  if (st != BNN_OK) return st;
  if (!aligned4(live)) return BNN_ERR_ALIGN;
  GatedActParams p = {};
  p.gu = gu, p.gu_ld = gu_ld, p.F = (int)F, p.act = act, p.live = live, p.q = q, p.q_ld = q_ld, p.scale = scale, p.scale_ld = scale_ld;
  return run_gated_act<GATE_F8>(p, type, S, static_cast<hipStream_t>(stream));
}

extern "C" bnn_status bnn_gated_act_backward(const void *gu, int type, int64_t S, int64_t gu_ld, int64_t F, int act, const int32_t *live,
                                             const void *dh, int64_t dh_ld, void *dgu, int64_t dgu_ld, void *stream) {
  using namespace bnn;
  const bnn_status st = check_gated_act(gu, type, S, gu_ld, F, act);
  if (st != BNN_OK) return st;
  if (dh_ld < F || dgu_ld < 2 * F) return BNN_ERR_STRIDE;
  if (S == 0) return BNN_OK;
  if (!dh || !dgu) return BNN_ERR_NULL;
  if (!aligned16(dh) || !aligned16(dgu) || !aligned4(live)) return BNN_ERR_ALIGN;
  GatedActParams p = {};
  p.gu = gu, p.gu_ld = gu_ld, p.F = (int)F, p.act = act, p.live = live, p.dh = dh, p.dh_ld = dh_ld, p.out = dgu, p.out_ld = dgu_ld;
  return run_gated_act<GATE_BACKWARD>(p, type, S, static_cast<hipStream_t>(stream));
}
