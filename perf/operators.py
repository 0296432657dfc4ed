"""Timed cases of the operators around 8-bit and gated layers: the int8 linear layer with a scale per token and output
channel, the norms after and before a block with the block's gate and residual scale, the gated feed-forward block with its
backward pass and its 8-bit form, and the sublayer that they make together.

`run` computes a case either by elementary torch operations in 32 bits (own = False) or through the entry points of
paper_1911_04477_amd.binding (own = True); both take the same state.  Widths are those of the fully-connected layers of
paper_1911_04477_amd.inputs and powers of two around them, token counts run from a single one to a long batch.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one token through a quantised fully-connected layer: the step of a served sequence, bound by the weights
        {"name": "linear_1x4096x4096", "kind": "linear", "M": 1, "N": 4096, "K": 4096, "type": "bf16", "bias": False},
        # the fully-connected layer of the workload configurations at its batch
        {"name": "linear_256x4096x4096", "kind": "linear", "M": 256, "N": 4096, "K": 4096, "type": "bf16", "bias": True},
        # off every tile edge, rows of no multiple of anything
        {"name": "linear_1000x3001_k2321", "kind": "linear", "M": 1000, "N": 3001, "K": 2321, "type": "f32", "bias": True},
        # a long prompt through wide layers
        {"name": "linear_8192x8192x8192", "kind": "linear", "M": 8192, "N": 8192, "K": 8192, "type": "bf16", "bias": False},
        # one token between two blocks: the smallest call of all
        {"name": "norm_1x4096", "kind": "norm", "T": 1, "D": 4096, "type": "bf16", "rtype": "bf16", "post": "rms",
         "pre": "rms", "gate": "channel", "scale": True, "train": False},
        # images of 250 tokens, each with a gate of its own; centred norms, fp32 residual stream, odd width
        {"name": "norm_1000x2321_groups", "kind": "norm", "T": 1000, "D": 2321, "type": "f16", "rtype": "f32",
         "post": "layer", "pre": "layer", "gate": "group", "scale": True, "train": False},
        # a training step over a batch of 8192 tokens: forward and backward, a gate for every token
        {"name": "norm_train_8192x4096", "kind": "norm", "T": 8192, "D": 4096, "type": "bf16", "rtype": "bf16",
         "post": "rms", "pre": "rms", "gate": "token", "scale": True, "train": True},
        # one token through the gated projections
        {"name": "gated_1_4096x8192", "kind": "gated", "T": 1, "D": 4096, "F": 8192, "type": "bf16", "act": "silu", "form": "plain"},
        # the 8-bit form at a serving batch, from floating-point activations
        {"name": "gated_i8_256_4096x8192", "kind": "gated", "T": 256, "D": 4096, "F": 8192, "type": "bf16", "act": "silu", "form": "i8"},
        # training on a ragged batch, odd hidden width, the other type and activation
        {"name": "gated_train_1000_1024x2321", "kind": "gated", "T": 1000, "D": 1024, "F": 2321, "type": "f16", "act": "gelu", "form": "train"},
        # training over a batch of 8192 tokens: the largest pass
        {"name": "gated_train_8192_4096x8192", "kind": "gated", "T": 8192, "D": 4096, "F": 8192, "type": "bf16", "act": "silu", "form": "train"},
        # the whole 8-bit sublayer for 64 sequences that are decoded together
        {"name": "block_64_4096x8192", "kind": "block", "T": 64, "D": 4096, "F": 8192, "type": "bf16", "act": "silu"},
    ]


# ---- drawn cases -----------------------------------------------------------------------------------------------------
MAX_LINEAR = 8192 ** 3
MAX_NORM = 8192 * 4096
MAX_GATED = 8192 * 4096 * 8192


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width of a layer: any, or a multiple of 64 as most have."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.5 else max(lo, w // 64 * 64)


def draw(rng):
    kind = rng.choice(["linear", "linear", "norm", "norm", "gated", "gated", "gated", "block"])
    while True:
        if kind == "linear":
            c = {"kind": kind, "M": _log_int(rng, 1, 8192), "N": _width(rng, 64, 16384), "K": _width(rng, 64, 16384),
                 "type": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.5}
            fits = c["M"] * c["N"] * c["K"] <= MAX_LINEAR
        elif kind == "norm":
            t = rng.choice(["bf16", "bf16", "f16", "f32"])
            c = {"kind": kind, "T": _log_int(rng, 1, 16384), "D": _width(rng, 64, 8192), "type": t,
                 "rtype": rng.choice([t, "f32"]), "post": rng.choice(["rms", "rms", "layer", "none"]),
                 "pre": rng.choice(["rms", "rms", "layer"]), "gate": rng.choice(["none", "channel", "group", "token"]),
                 "scale": rng.random() < 0.7, "train": rng.random() < 0.5}
            fits = c["T"] * c["D"] * (2 if t == "f32" or c["rtype"] == "f32" else 1) <= MAX_NORM
        else:
            c = {"kind": kind, "T": _log_int(rng, 1, 8192), "D": _width(rng, 64, 8192), "F": _width(rng, 64, 16384),
                 "type": rng.choice(["bf16", "bf16", "f16"]), "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])}
            if kind == "gated":
                c["form"] = rng.choice(["plain", "i8", "train"])
            fits = c["T"] * c["D"] * c["F"] <= MAX_GATED
        if fits:
            return c


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _pad16(n):
    return (n + 15) // 16 * 16


def _activations(g, T, D, dtype):
    """Normal values, a few channels much larger than the others."""
    x = torch.randn((T, D), generator=g, device=DEV)
    x *= torch.where(torch.rand((D,), generator=g, device=DEV) < 0.01, 8.0, 1.0)
    return x.to(dtype)


def _weight_i8(g, N, K):
    """An 8-bit weight as it is kept between calls: rows that start on 16 bytes, one scale per output channel."""
    w = torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K)
    s = w.abs().amax(1) / 127
    q = torch.zeros((N, _pad16(K)), dtype=torch.int8, device=DEV)[:, :K]
    q.copy_((w / s[:, None]).round().clamp(-127, 127))
    return q, s


def _rows_i8(T, K):
    """Room for 8-bit activations."""
    return torch.zeros((T, _pad16(K)), dtype=torch.int8, device=DEV)[:, :K], torch.zeros((T,), device=DEV)


def _norm_inputs(c, g):
    T, D, dt, rt = c["T"], c["D"], TYPES[c["type"]], TYPES[c["rtype"]]

    def vec(mean, std):
        return mean + std * torch.randn((D,), generator=g, device=DEV)

    group = {"none": 0, "channel": T, "group": max(1, (T + 3) // 4), "token": 1}[c["gate"]]
    s = {"b": (0.5 * _activations(g, T, D, torch.float32) + (0.3 if c["post"] == "layer" else 0.0)).to(dt),
         "r": (2 * torch.randn((T, D), generator=g, device=DEV)).to(rt), "gate_rows": group, "gate": None, "res_scale": None,
         "w_post": None, "bias_post": None, "w_pre": None, "bias_pre": None, "post": c["post"], "pre": c["pre"]}
    if group:
        s["gate"] = (0.5 + 0.3 * torch.randn(((T + group - 1) // group, D), generator=g, device=DEV)).to(dt)
    if c["scale"]:
        s["res_scale"] = vec(0.5, 0.1)
    for which in ("post", "pre"):
        if c[which] != "none":
            s["w_" + which] = vec(1.0, 0.1)
        if c[which] == "layer":
            s["bias_" + which] = vec(0.0, 0.1)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    c, dt = case, TYPES[case["type"]]
    s = {"case": c}
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = _activations(g, M, K, dt)
        s["w"], s["ws"] = _weight_i8(g, N, K)
        s["bias"] = 0.1 * torch.randn((N,), generator=g, device=DEV) if c["bias"] else None
        s["q"], s["qs"] = _rows_i8(M, K)
        s["y"] = torch.empty((M, N), dtype=dt, device=DEV)
    elif c["kind"] == "norm":
        s.update(_norm_inputs(c, g))
        s["r_out"], s["n_out"] = torch.empty_like(s["r"]), torch.empty_like(s["b"])
        if c["train"]:
            s["dn"] = torch.randn((c["T"], c["D"]), generator=g, device=DEV).to(dt)
            s["dr_out"] = torch.randn((c["T"], c["D"]), generator=g, device=DEV).to(s["r"].dtype)
    elif c["kind"] == "gated":
        T, D, F = c["T"], c["D"], c["F"]
        s["x"] = _activations(g, T, D, dt)
        if c["form"] == "i8":
            (s["wg"], s["sg"]), (s["wu"], s["su"]) = _weight_i8(g, F, D), _weight_i8(g, F, D)
            s["q"], s["qs"] = _rows_i8(T, D)
        else:
            s["wg"], s["wu"] = ((torch.randn((F, D), generator=g, device=DEV) / math.sqrt(D)).to(dt) for _ in range(2))
        s["h"] = torch.empty((T, F), dtype=dt, device=DEV)
        if c["form"] == "train":
            s["dh"] = torch.randn((T, F), generator=g, device=DEV).to(dt)
    else:
        T, D, F = c["T"], c["D"], c["F"]
        s.update(_norm_inputs({**c, "rtype": c["type"], "post": "rms", "pre": "rms", "gate": "channel", "scale": True}, g))
        (s["wg"], s["sg"]), (s["wu"], s["su"]), (s["wd"], s["sd"]) = _weight_i8(g, F, D), _weight_i8(g, F, D), _weight_i8(g, D, F)
        s["q"], s["qs"] = _rows_i8(T, D)
        s["qh"], s["qhs"] = _rows_i8(T, F)
        s["h"] = torch.empty((T, F), dtype=dt, device=DEV)
        s["o"], s["n_out"], s["r1"], s["r2"] = (torch.empty((T, D), dtype=dt, device=DEV) for _ in range(4))
    return s


# ---- the operators in plain form: 32 bits, rounded once at the end -----------------------------------------------------
def _plain_quant(x):
    x = x.float()
    a = x.abs().amax(1, keepdim=True)
    some = a >= 2.0 ** -100
    full = torch.full_like(a, 127.0)
    inv = torch.where(some, full / a, torch.zeros_like(a))
    return (x * inv).round().clamp(-127, 127), torch.where(some, a / full, torch.zeros_like(a))


def _plain_product(q, qs, w, ws):
    return (q.float() @ w.float().T) * qs * ws


def _plain_linear(x, w, ws, bias, dt):
    q, qs = _plain_quant(x)
    y = _plain_product(q, qs, w, ws)
    return (y if bias is None else y + bias).to(dt)


def _plain_act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return torch.relu(z)


def _plain_act_slope(z, act):
    if act == "silu":
        t = torch.sigmoid(z)
        return t * (1 + z * (1 - t))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    return (z > 0).to(z.dtype)


def _plain_unit(x, norm):
    """The normed rows before weight and bias, and the factor of each row."""
    if norm == "none":
        return x, None
    if norm == "layer":
        x = x - x.mean(1, keepdim=True)
    rs = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * rs, rs


def _plain_affine(x, w, bias):
    x = x if w is None else x * w
    return x if bias is None else x + bias


def _plain_factor(s):
    """What a block's normed output is multiplied with on its way into the residual stream: [T, D], [D] or 1."""
    m = torch.ones((), device=DEV) if s["res_scale"] is None else s["res_scale"]
    if s["gate"] is not None:
        m = m * s["gate"].float().repeat_interleave(s["gate_rows"], 0)[: s["b"].shape[0]]
    return m


def _plain_norm(s):
    p = _plain_affine(_plain_unit(s["b"].float(), s["post"])[0], s["w_post"], s["bias_post"])
    r1 = s["r"].float() + _plain_factor(s) * p
    return r1, _plain_affine(_plain_unit(r1, s["pre"])[0], s["w_pre"], s["bias_pre"])


def _plain_unit_backward(e, u, rs, norm):
    if norm == "none":
        return e
    if norm == "layer":
        e = e - e.mean(1, keepdim=True)
    return rs * (e - u * (e * u).mean(1, keepdim=True))


def _plain_norm_backward(s):
    m = _plain_factor(s)
    ub, rsb = _plain_unit(s["b"].float(), s["post"])
    p = _plain_affine(ub, s["w_post"], s["bias_post"])
    ur, rsr = _plain_unit(s["r"].float() + m * p, s["pre"])
    dn = s["dn"].float()
    e = dn if s["w_pre"] is None else dn * s["w_pre"]
    dr = s["dr_out"].float() + _plain_unit_backward(e, ur, rsr, s["pre"])
    dp = dr * m
    e = dp if s["w_post"] is None else dp * s["w_post"]
    got = {"dr": dr.to(s["r"].dtype), "db": _plain_unit_backward(e, ub, rsb, s["post"]).to(s["b"].dtype)}
    if s["w_pre"] is not None:
        got["dw_pre"] = (dn * ur).sum(0)
    if s["bias_pre"] is not None:
        got["dbias_pre"] = dn.sum(0)
    if s["w_post"] is not None:
        got["dw_post"] = (dp * ub).sum(0)
    if s["bias_post"] is not None:
        got["dbias_post"] = dp.sum(0)
    if s["res_scale"] is not None:
        t = dr * p
        if s["gate"] is not None:
            t = t * s["gate"].float().repeat_interleave(s["gate_rows"], 0)[: dr.shape[0]]
        got["dres_scale"] = t.sum(0)
    if s["gate"] is not None:
        t = dr * p
        t = t if s["res_scale"] is None else t * s["res_scale"]
        n = s["gate"].shape[0] * s["gate_rows"] - t.shape[0]
        t = torch.cat([t, t.new_zeros((n, t.shape[1]))]) if n else t
        got["dgate"] = t.reshape(s["gate"].shape[0], s["gate_rows"], -1).sum(1).to(s["gate"].dtype)
    return got


def _plain_gated(s, dt):
    c = s["case"]
    if c["form"] == "i8":
        q, qs = _plain_quant(s["x"])
        g, u = _plain_product(q, qs, s["wg"], s["sg"]), _plain_product(q, qs, s["wu"], s["su"])
    else:
        x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
        g, u = x @ wg.T, x @ wu.T
    a = _plain_act(g, c["act"])
    h = (a * u).to(dt)
    if c["form"] != "train":
        return h
    dh = s["dh"].float()
    dg, du = dh * u * _plain_act_slope(g, c["act"]), dh * a
    return {"h": h, "dx": (dg @ wg + du @ wu).to(dt), "dwg": (dg.T @ x).to(dt), "dwu": (du.T @ x).to(dt)}


def _plain_block(s, dt):
    """Operator after operator, each rounded at its own end."""
    r1, n1 = _plain_norm(s)
    r1 = r1.to(dt)
    q, qs = _plain_quant(n1)
    g, u = _plain_product(q, qs, s["wg"], s["sg"]), _plain_product(q, qs, s["wu"], s["su"])
    h = (_plain_act(g, s["case"]["act"]) * u).to(dt)
    o = _plain_linear(h, s["wd"], s["sd"], None, dt)
    r2, n2 = _plain_norm({**s, "b": o, "r": r1})
    return {"r1": r1, "h": h, "r2": r2.to(dt), "n": n2.to(dt)}


def run(state):
    s, c = state, state["case"]
    dt = TYPES[c["type"]]
    if own:
        return _run_own(s, c)
    if c["kind"] == "linear":
        return _plain_linear(s["x"], s["w"], s["ws"], s["bias"], dt)
    if c["kind"] == "norm":
        r1, n = _plain_norm(s)
        got = {"r": r1.to(s["r"].dtype), "n": n.to(dt)}
        return {**got, **_plain_norm_backward(s)} if c["train"] else got
    return _plain_gated(s, dt) if c["kind"] == "gated" else _plain_block(s, dt)


# ---- the same through the framework's operators ------------------------------------------------------------------------
def _run_own(s, c):
    from paper_1911_04477_amd import binding as B

    if c["kind"] == "linear":
        B.bnn_quant_rows_i8(s["x"], s["q"], s["qs"])
        return B.bnn_linear_i8(s["q"], s["qs"], s["w"], s["ws"], s["bias"], out=s["y"])
    if c["kind"] == "norm":
        given = dict(gate=s["gate"], gate_rows=s["gate_rows"], res_scale=s["res_scale"], w_post=s["w_post"],
                     bias_post=s["bias_post"], w_pre=s["w_pre"], bias_pre=s["bias_pre"], post=s["post"], pre=s["pre"], eps=EPS)
        r1, n = B.bnn_norm_gate(s["b"], s["r"], r_out=s["r_out"], n_out=s["n_out"], **given)
        if not c["train"]:
            return {"r": r1, "n": n}
        return {"r": r1, "n": n, **B.bnn_norm_gate_backward(s["b"], s["r"], s["dn"], s["dr_out"], **given)}
    if c["kind"] == "gated":
        if c["form"] == "i8":
            B.bnn_quant_rows_i8(s["x"], s["q"], s["qs"])
            return B.bnn_gated_ff_i8(s["q"], s["qs"], s["wg"], s["sg"], s["wu"], s["su"], act=c["act"], out=s["h"])
        if c["form"] == "plain":
            return B.bnn_gated_ff(s["x"], s["wg"], s["wu"], act=c["act"], out=s["h"])
        saved = B.gated_ff_saved(c["T"], c["F"], s["x"].device)
        h = B.bnn_gated_ff(s["x"], s["wg"], s["wu"], act=c["act"], out=s["h"], saved=saved)
        dx, dwg, dwu = B.bnn_gated_ff_backward(s["x"], s["wg"], s["wu"], saved, s["dh"])
        return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}
    given = dict(gate=s["gate"], gate_rows=s["gate_rows"], res_scale=s["res_scale"], w_post=s["w_post"], w_pre=s["w_pre"],
                 post="rms", pre="rms", eps=EPS)
    B.bnn_norm_gate(s["b"], s["r"], r_out=s["r1"], q_out=s["q"], q_scale=s["qs"], **given)
    B.bnn_gated_ff_i8(s["q"], s["qs"], s["wg"], s["sg"], s["wu"], s["su"], act=c["act"], out=s["h"])
    B.bnn_quant_rows_i8(s["h"], s["qh"], s["qhs"])
    B.bnn_linear_i8(s["qh"], s["qhs"], s["wd"], s["sd"], out=s["o"])
    B.bnn_norm_gate(s["o"], s["r1"], r_out=s["r2"], n_out=s["n_out"], **given)
    return {"r1": s["r1"], "h": s["h"], "r2": s["r2"], "n": s["n_out"]}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    c, size = case, TYPES[case["type"]].itemsize
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": M * K * size + N * K + 4 * N * (2 if c["bias"] else 1) + M * N * size, "flops": 2 * M * N * K}
    if c["kind"] == "norm":
        T, D, rsize = c["T"], c["D"], TYPES[c["rtype"]].itemsize
        gates = {"none": 0, "channel": 1, "group": min(T, 4), "token": T}[c["gate"]] * D * size
        vectors = 4 * D * (c["scale"] + {"none": 0, "rms": 1, "layer": 2}[c["post"]] + {"none": 0, "rms": 1, "layer": 2}[c["pre"]])
        w = {"bytes": 2 * T * D * (size + rsize) + gates + vectors, "flops": 12 * T * D}
        if c["train"]:  # b, r, their gates and vectors are read once; dn, dr_out come in, dr, db and the sums go out
            w = {"bytes": w["bytes"] + 2 * T * D * (size + rsize) + gates + vectors, "flops": 40 * T * D}
        return w
    T, D, F = c["T"], c["D"], c["F"]
    if c["kind"] == "block":
        return {"bytes": 5 * T * D * size + T * F * size + 3 * D * F + 8 * F + 4 * D + D * size + 12 * D, "flops": 6 * T * D * F}
    if c["form"] == "i8":
        return {"bytes": T * D * size + 2 * F * D + 8 * F + T * F * size, "flops": 4 * T * D * F}
    if c["form"] == "plain":
        return {"bytes": (T * D + 2 * F * D + T * F) * size, "flops": 4 * T * D * F}
    return {"bytes": (2 * T * D + 4 * F * D + 2 * T * F) * size, "flops": 12 * T * D * F}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
class _Exact:
    """Each operator from its formula, row statistics and products in 64 bits."""

    @staticmethod
    def rows_i8(x):
        x = x.double()
        top = x.abs().max(dim=1, keepdim=True).values
        step = torch.where(top >= 2.0 ** -100, top / 127.0, torch.zeros_like(top))
        q = torch.where(step > 0, torch.round(x / step.clamp(min=1e-300)), torch.zeros_like(x))
        return q, step

    @staticmethod
    def matmul_i8(q, step, w, ws):
        return torch.mm(q, w.double().t()).mul_(step).mul_(ws.double())

    @staticmethod
    def act(z, name):
        """The activation and its derivative."""
        if name == "silu":
            t = 1.0 / (1.0 + torch.exp(-z))
            return z * t, t + z * t * (1.0 - t)
        if name == "gelu":
            cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
            return z * cdf, cdf + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
        if name == "gelu_tanh":
            a, k = math.sqrt(2.0 / math.pi), 0.044715
            t = torch.tanh(a * z * (1.0 + k * z * z))
            return z * (1.0 + t) / 2.0, (1.0 + t) / 2.0 + z * (1.0 - t * t) * a * (1.0 + 3.0 * k * z * z) / 2.0
        return torch.clamp(z, min=0.0), torch.gt(z, 0).double()

    @staticmethod
    def unit(x, norm):
        if norm == "none":
            return x, torch.ones_like(x[:, :1])
        x = x - x.mean(dim=1, keepdim=True) if norm == "layer" else x
        sd = torch.sqrt(x.square().sum(dim=1, keepdim=True) / x.shape[1] + EPS)
        return x / sd, 1.0 / sd

    @staticmethod
    def unit_grad(e, u, inv, norm):
        if norm == "none":
            return e
        n = e.shape[1]
        along = u * ((e * u).sum(dim=1, keepdim=True) / n)
        level = e.sum(dim=1, keepdim=True) / n if norm == "layer" else 0.0
        return (e - level - along) * inv

    def norm(self, s, grad):
        T, D = s["b"].shape
        one = torch.ones((D,), dtype=torch.float64, device=DEV)

        def of(name):
            return one if s[name] is None else s[name].double()

        zero = one * 0
        bias_post = zero if s["bias_post"] is None else s["bias_post"].double()
        bias_pre = zero if s["bias_pre"] is None else s["bias_pre"].double()
        if s["gate"] is None:
            gate = one[None]
        else:
            gate = s["gate"].double()[torch.arange(T, device=DEV) // s["gate_rows"]]
        ub, ib = self.unit(s["b"].double(), s["post"])
        p = ub * of("w_post") + bias_post
        r1 = s["r"].double() + of("res_scale") * gate * p
        ur, ir = self.unit(r1, s["pre"])
        got = {"r": r1, "n": ur * of("w_pre") + bias_pre}
        if not grad:
            return got
        dn = s["dn"].double()
        dr = s["dr_out"].double() + self.unit_grad(dn * of("w_pre"), ur, ir, s["pre"])
        dp = dr * of("res_scale") * gate
        got.update(dr=dr, db=self.unit_grad(dp * of("w_post"), ub, ib, s["post"]))
        sums = {"w_pre": dn * ur, "bias_pre": dn, "w_post": dp * ub, "bias_post": dp, "res_scale": dr * gate * p}
        got.update({"d" + k: v.sum(dim=0) for k, v in sums.items() if s[k] is not None})
        if s["gate"] is not None:
            got["dgate"] = torch.zeros_like(s["gate"], dtype=torch.float64).index_add_(
                0, torch.arange(T, device=DEV) // s["gate_rows"], dr * of("res_scale") * p)
        return got

    def gated(self, s, c):
        if c["form"] == "i8":
            q, step = self.rows_i8(s["x"])
            g, u = self.matmul_i8(q, step, s["wg"], s["sg"]), self.matmul_i8(q, step, s["wu"], s["su"])
            return self.act(g, c["act"])[0] * u
        x, wg, wu = s["x"].double(), s["wg"].double(), s["wu"].double()
        g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        a, slope = self.act(g, c["act"])
        if c["form"] == "plain":
            return a * u
        dh = s["dh"].double()
        dg, du = dh * u * slope, dh * a
        return {"h": a * u, "dx": torch.mm(dg, wg) + torch.mm(du, wu), "dwg": torch.mm(dg.t(), x), "dwu": torch.mm(du.t(), x)}

    def block(self, s, c, dt):
        """The sublayer's definition has its intermediate values in the tensors' type: r1, h and o are rounded to it."""
        first = self.norm(s, False)
        q, step = self.rows_i8(first["n"])
        g, u = self.matmul_i8(q, step, s["wg"], s["sg"]), self.matmul_i8(q, step, s["wu"], s["su"])
        h = self.act(g, c["act"])[0] * u
        q, step = self.rows_i8(h.to(dt))
        last = self.norm({**s, "b": self.matmul_i8(q, step, s["wd"], s["sd"]).to(dt), "r": first["r"].to(dt)}, False)
        return {"r1": first["r"], "h": h, "r2": last["r"], "n": last["n"]}


def exact(case, seed):
    s, c, E = prepare(case, seed), case, _Exact()
    if c["kind"] == "linear":
        q, step = E.rows_i8(s["x"])
        y = E.matmul_i8(q, step, s["w"], s["ws"])
        return y if s["bias"] is None else y + s["bias"].double()
    if c["kind"] == "norm":
        return E.norm(s, c["train"])
    return E.gated(s, c) if c["kind"] == "gated" else E.block(s, c, TYPES[c["type"]])
