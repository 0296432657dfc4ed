"""A gated feed-forward sublayer of a residual network as a sequence of C-ABI calls (orchestration only).

    r', n  = norm_gate(b, r)            the block before is normed, gated and scaled into the stream; n is the stream's norm
    h      = act(n Wg^T) * (n Wu^T)
    o      = h Wd^T                     what the next norm_gate takes as its b

GatedBlock8 is the serving form: weights and activations in 8 bits with a scale per output channel and per token, any
number of tokens from one to the number it was made for, nothing allocated in a pass that is given r_out (it can be captured in a graph).  Its
buffers serve one pass at a time: threads or streams that run at once need an object each.
GatedProjections is the training form of the part that has a backward pass: the norms and both projections.

The same with experts, in 8-bit floating point: each token's rows go to the experts chosen for it and come back weighted.

    xs = rows of x sorted by expert,  gu = xs W1_e^T,  h = act(g) * u,  ys = h W2_e^T,  out[t] = sum over its experts of weight * ys

ExpertBlock8 serves it (weights quantised once, buffers made once), ExpertLayer trains it.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from . import binding as B


class GatedBlock8:
    """wg, wu [F, D], wd [D, F]: fp32, bf16 or fp16, quantized here once.  vectors: the keyword arguments of bnn_norm_gate that
    hold parameters (res_scale, w_post, bias_post, w_pre, bias_pre, post, pre, eps).  A pass writes the 8-bit rows, their scales, h and o
    of the pass before over."""

    def __init__(self, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor, tokens: int, vectors: Optional[Dict] = None,
                 act: str = "silu", dtype: torch.dtype = torch.bfloat16):
        (self.F, self.D), self.act, self.tokens = wg.shape, act, tokens
        self.vectors = dict(vectors or {})
        self.wg, self.wu, self.wd = (B.bnn_quant_rows_i8(w) for w in (wg, wu, wd))
        dev = wg.device
        self.n8, self.n_scale = B.rows_i8(tokens, self.D, dev), torch.empty((tokens,), dtype=torch.float32, device=dev)
        self.h8, self.h_scale = B.rows_i8(tokens, self.F, dev), torch.empty((tokens,), dtype=torch.float32, device=dev)
        self.h = torch.empty((tokens, self.F), dtype=dtype, device=dev)
        self.o = torch.empty((tokens, self.D), dtype=dtype, device=dev)

    def forward(self, b: Optional[torch.Tensor], r: torch.Tensor, gate: Optional[torch.Tensor] = None, gate_rows: int = 1,
                r_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """b: the output of the block before (None before the first), r: the stream, both [T, D] -> (o, r'), o in a buffer that
        the next pass writes again.  r_out may be r; without b the stream stays r."""
        T = r.shape[0]
        if T > self.tokens:
            raise ValueError(f"made for {self.tokens} tokens")
        n8, n_scale, h, h8, h_scale, o = (t[:T] for t in (self.n8, self.n_scale, self.h, self.h8, self.h_scale, self.o))
        given = dict(self.vectors)
        if b is None:
            given = {k: v for k, v in given.items() if k in ("w_pre", "bias_pre", "pre", "eps")}
            given["post"] = "none"
        r1, _ = B.bnn_norm_gate(b, r, gate=gate, gate_rows=gate_rows, r_out=r_out, q_out=n8, q_scale=n_scale, **given)
        B.bnn_gated_ff_i8(n8, n_scale, *self.wg, *self.wu, act=self.act, out=h)
        B.bnn_quant_rows_i8(h, h8, h_scale)
        B.bnn_linear_i8(h8, h_scale, *self.wd, out=o)
        return o, r if b is None else r1


class GatedProjections:
    """wg, wu [F, D] and the parameters of the norms; forward keeps what backward needs, for one pass at a time."""

    def __init__(self, wg: torch.Tensor, wu: torch.Tensor, vectors: Optional[Dict] = None, act: str = "silu"):
        self.wg, self.wu, self.vectors, self.act = wg, wu, dict(vectors or {}), act
        self.kept: Optional[Tuple] = None

    def forward(self, b: torch.Tensor, r: torch.Tensor, gate: Optional[torch.Tensor] = None,
                gate_rows: int = 1) -> Tuple[torch.Tensor, torch.Tensor]:
        """b, r [T, D] -> (h [T, F], r' [T, D])."""
        given = dict(self.vectors, gate=gate, gate_rows=gate_rows)
        r1, n = B.bnn_norm_gate(b, r, **given)
        saved = B.gated_ff_saved(r.shape[0], self.wg.shape[0], r.device)
        h = B.bnn_gated_ff(n, self.wg, self.wu, act=self.act, saved=saved)
        self.kept = (b, r, n, saved, given)
        return h, r1

    def backward(self, dh: torch.Tensor, dr_out: Optional[torch.Tensor]) -> Dict[str, torch.Tensor]:
        """Gradients of the last forward pass from those of h and of r' (None: zero): db, dr, dwg, dwu and those of the norms'
        parameters and the gate that it was given."""
        if self.kept is None:
            raise RuntimeError("backward comes after a forward pass of its own")
        (b, r, n, saved, given), self.kept = self.kept, None
        dn, dwg, dwu = B.bnn_gated_ff_backward(n, self.wg, self.wu, saved, dh)
        return {"dwg": dwg, "dwu": dwu, **B.bnn_norm_gate_backward(b, r, dn, dr_out, **given)}


def _choices(x: torch.Tensor, experts: torch.Tensor) -> Tuple[int, int]:
    """Tokens and choices of each.  Slots of tokens that x does not have would be left as they were, without an error of their own."""
    if x.dim() != 2 or experts.dim() != 2 or x.shape[0] != experts.shape[0]:
        raise ValueError(f"x [T, D] and experts [T, choices] expected, got {list(x.shape)} and {list(experts.shape)}")
    return experts.shape[0], experts.shape[1]


class ExpertBlock8:
    """w1 [E, 2 F, D] (gate and up projections one below the other), w2 [E, D, F]: fp32, bf16 or fp16, quantised here once to e4m3
    in blocks of 128 x 128.  Any number of tokens from one to `tokens`, `choices` experts each; a pass allocates nothing where it is
    given out (it can be captured in a graph), and writes the buffers of the pass before over: threads or streams that run at once need
    an object each.  fast: products with fast sums, of bf16 only (B.bnn_linear_f8)."""

    def __init__(self, w1: torch.Tensor, w2: torch.Tensor, tokens: int, choices: int, act: str = "silu",
                 dtype: torch.dtype = torch.bfloat16, fast: bool = False):
        (self.E, self.D, self.F), self.act, self.tokens, self.choices, self.fast = w2.shape, act, tokens, choices, fast
        if w1.shape != (self.E, 2 * self.F, self.D):
            raise ValueError(f"w1: [{self.E}, {2 * self.F}, {self.D}] expected")
        if fast and dtype != torch.bfloat16:
            raise ValueError("fast: sums of bf16 only")
        (self.w1, _), (self.w2, _) = (B.bnn_quant_weight_f8(w, turned=False) for w in (w1, w2))
        dev, S = w1.device, tokens * choices
        self.offsets = torch.empty((self.E + 1,), dtype=torch.int32, device=dev)
        self.rows, self.places = (torch.empty((S,), dtype=torch.int32, device=dev) for _ in range(2))
        self.workspace = torch.empty((B.expert_sort_workspace_bytes(tokens, choices, self.E),), dtype=torch.uint8, device=dev)
        self.x8, self.x_scale = B.rows_f8(S, self.D, dev), B.scales_f8(S, self.D, dev)
        self.h8, self.h_scale = B.rows_f8(S, self.F, dev), B.scales_f8(S, self.F, dev)
        self.gu, self.ys = (torch.empty((S, n), dtype=dtype, device=dev) for n in (2 * self.F, self.D))

    def forward(self, x: torch.Tensor, experts: torch.Tensor, weights: torch.Tensor,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [T, D], experts [T, choices] int32 or int64 (outside 0 .. E - 1: none), weights [T, choices] fp32 -> [T, D]."""
        T, k = _choices(x, experts)
        if T > self.tokens or k != self.choices:
            raise ValueError(f"made for {self.tokens} tokens of {self.choices} choices")
        S = T * k
        x8, x_scale, h8, h_scale, gu, ys = (t[:S] for t in (self.x8, self.x_scale, self.h8, self.h_scale, self.gu, self.ys))
        offsets, rows, places = B.bnn_expert_sort(experts, self.E, offsets=self.offsets, rows=self.rows[:S],
                                                  places=self.places[:S].view(T, k), workspace=self.workspace)
        B.bnn_quant_blocks_f8(x, x8, x_scale, rows=rows, k=k)
        B.bnn_expert_linear_f8(x8, x_scale, offsets, *self.w1, out=gu, fast=self.fast)
        B.bnn_gated_act_f8(gu, act=self.act, q=h8, scale=h_scale)
        B.bnn_expert_linear_f8(h8, h_scale, offsets, *self.w2, out=ys, fast=self.fast)
        return B.bnn_expert_combine(ys, places, weights, out=out)


class ExpertLayer:
    """w1 [E, 2 F, D], w2 [E, D, F]; products in e4m3 with block scales, everything between them in the tensors' type.  Weights are
    quantised anew in each forward pass, which keeps what backward needs, for one pass at a time.  fast: products of rows with fast sums,
    of bf16 only (B.bnn_linear_f8); the weights' gradients are fp32's always."""

    def __init__(self, w1: torch.Tensor, w2: torch.Tensor, act: str = "silu", fast: bool = False):
        self.w1, self.w2, self.act, self.fast = w1, w2, act, fast
        self.kept: Optional[Tuple] = None

    def forward(self, x: torch.Tensor, experts: torch.Tensor, weights: torch.Tensor) -> torch.Tensor:
        """x [T, D], experts [T, k], weights [T, k] fp32 -> [T, D]."""
        _, k = _choices(x, experts)
        offsets, rows, places = B.bnn_expert_sort(experts, self.w2.shape[0], align=B.F8_BLOCK)
        (w1, w1t), (w2, w2t) = B.bnn_quant_weight_f8(self.w1), B.bnn_quant_weight_f8(self.w2)
        gu = B.bnn_expert_linear_f8(*B.bnn_quant_blocks_f8(x, rows=rows, k=k), offsets, *w1, dtype=x.dtype, fast=self.fast)
        h8 = B.bnn_gated_act_f8(gu, act=self.act, live=offsets[-1:])
        ys = B.bnn_expert_linear_f8(*h8, offsets, *w2, dtype=x.dtype, fast=self.fast)
        self.kept = (x, k, offsets, rows, places, weights, w1t, w2t, gu, ys)
        return B.bnn_expert_combine(ys, places, weights)

    def backward(self, dout: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Gradients of the last forward pass from that of its output: dx, dweights [T, k], dw1 and dw2 (fp32)."""
        if self.kept is None:
            raise RuntimeError("backward comes after a forward pass of its own")
        (x, k, offsets, rows, places, weights, w1t, w2t, gu, ys), self.kept = self.kept, None
        live = offsets[-1:]
        dys, dweights = B.bnn_expert_combine_backward(ys, rows, places, weights, dout)
        dh = B.bnn_expert_linear_f8(*B.bnn_quant_blocks_f8(dys), offsets, *w2t, dtype=x.dtype, fast=self.fast)
        h = B.bnn_gated_act(gu, act=self.act, live=live)
        dw2 = B.bnn_expert_linear_f8_dw(*B.bnn_quant_columns_f8(dys), *B.bnn_quant_columns_f8(h), offsets)
        dgu = B.bnn_gated_act_backward(gu, dh, act=self.act, live=live)
        dw1 = B.bnn_expert_linear_f8_dw(*B.bnn_quant_columns_f8(dgu), *B.bnn_quant_columns_f8(x, rows=rows, k=k), offsets)
        dxs = B.bnn_expert_linear_f8(*B.bnn_quant_blocks_f8(dgu), offsets, *w1t, dtype=x.dtype, fast=self.fast)
        return {"dx": B.bnn_expert_combine(dxs, places), "dweights": dweights, "dw1": dw1, "dw2": dw2}
