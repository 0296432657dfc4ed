"""A gated feed-forward sublayer of a residual network as a sequence of C-ABI calls (orchestration only).

    r', n  = norm_gate(b, r)            the block before is normed, gated and scaled into the stream; n is the stream's norm
    h      = act(n Wg^T) * (n Wu^T)
    o      = h Wd^T                     what the next norm_gate takes as its b

GatedBlock8 is the serving form: weights and activations in 8 bits with a scale per output channel and per token, any
number of tokens from one to the number it was made for, nothing allocated in a pass that is given r_out (it can be captured in a graph).  Its
buffers serve one pass at a time: threads or streams that run at once need an object each.
GatedProjections is the training form of the part that has a backward pass: the norms and both projections.
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
