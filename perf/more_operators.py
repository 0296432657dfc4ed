"""Timed cases of the operators around 8-bit floating point and experts: the linear layer on e4m3 values with a scale for each
block of 128 of them, tokens sorted by expert and back with weights, the experts' products, the gated activation that feeds the
second of them, with the gradients of all, and the expert layer that they make together.

`run` computes a case either by elementary torch operations in 32 bits (own = False) or through the entry points of
paper_1911_04477_amd.binding (own = True); both take the same state.  Widths are those of the fully-connected layers of
paper_1911_04477_amd.inputs and powers of two around them, token counts run from a single one to a long batch.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 128


def listed():
    return [
        # one token through a linear layer: the step of a served sequence, bound by the weights
        {"name": "linear_1x4096x4096", "kind": "linear", "M": 1, "N": 4096, "K": 4096, "type": "bf16", "scales": "pow2",
         "bias": False, "train": False},
        # off every tile edge, weights with fp32 scales from elsewhere
        {"name": "linear_1000x3001_k2321", "kind": "linear", "M": 1000, "N": 3001, "K": 2321, "type": "f32", "scales": "f32",
         "bias": True, "train": False},
        # a training step of a linear layer over 8192 tokens, weights and gradients in 16 bits outside of the products
        {"name": "linear_train_8192_4096x4096", "kind": "linear", "M": 8192, "N": 4096, "K": 4096, "type": "bf16",
         "scales": "pow2", "bias": False, "train": True},
        # one token to 8 of 64 experts and back: the smallest call of all
        {"name": "route_1x8_of_64", "kind": "route", "T": 1, "k": 8, "E": 64, "D": 4096, "type": "bf16", "align": 1,
         "drop": False, "train": False},
        # a ragged batch of odd width, some tokens refused by their expert
        {"name": "route_1000x3_of_17_drop", "kind": "route", "T": 1000, "k": 3, "E": 17, "D": 2321, "type": "f16", "align": 1,
         "drop": True, "train": True},
        # a training step over 8192 tokens, experts' rows in whole blocks of 128 as their weights' gradients need them
        {"name": "route_train_8192x4_of_64", "kind": "route", "T": 8192, "k": 4, "E": 64, "D": 4096, "type": "bf16",
         "align": 128, "drop": False, "train": True},
        # sixteen sequences decoded together: few rows an expert
        {"name": "experts_16x2_of_8_4096x8192", "kind": "experts", "T": 16, "k": 2, "E": 8, "K": 4096, "N": 8192,
         "type": "bf16", "align": 1, "train": False},
        # training on a ragged batch, odd hidden width, few experts
        {"name": "experts_train_1000x2_of_5_1024x2321", "kind": "experts", "T": 1000, "k": 2, "E": 5, "K": 1024, "N": 2321,
         "type": "f16", "align": 128, "train": True},
        # experts' hidden values of a ragged prompt on their way into the second product
        {"name": "gate_1000x2321", "kind": "gate", "S": 1000, "F": 2321, "type": "f16", "act": "gelu", "train": False},
        # the same of a training batch, with its gradient
        {"name": "gate_train_16384x4096", "kind": "gate", "S": 16384, "F": 4096, "type": "bf16", "act": "silu", "train": True},
        # one token through a whole expert layer
        {"name": "block_1x8_of_64_2048x1024", "kind": "block", "T": 1, "k": 8, "E": 64, "D": 2048, "F": 1024, "type": "bf16",
         "act": "silu"},
        # a prompt of 4096 tokens through it
        {"name": "block_4096x2_of_8_2048x4096", "kind": "block", "T": 4096, "k": 2, "E": 8, "D": 2048, "F": 4096,
         "type": "bf16", "act": "silu"},
    ]


# ---- drawn cases -----------------------------------------------------------------------------------------------------
MAX_LINEAR = 3 * 8192 * 4096 * 4096      # multiply-adds of all products of a pass
MAX_WEIGHTS = 8 * 3 * 2048 * 4096
MAX_ROUTE = 8192 * 4 * 4096
MAX_GATE = 16384 * 4096


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width of a layer: any, or a multiple of 64 as most have."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.5 else max(lo, w // 64 * 64)


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "route", "route", "experts", "experts", "experts", "gate", "block", "block"])
    while True:
        train, dtype = rng.random() < 0.5, rng.choice(["bf16", "bf16", "f16", "f32"])
        if kind == "linear":
            c = {"kind": kind, "M": _log_int(rng, 1, 8192), "N": _width(rng, 64, 16384), "K": _width(rng, 64, 16384),
                 "type": dtype, "scales": "pow2" if train else rng.choice(["pow2", "f32"]), "bias": rng.random() < 0.5,
                 "train": train}
            fits = c["M"] * c["N"] * c["K"] * (3 if train else 1) <= MAX_LINEAR
        elif kind == "gate":
            c = {"kind": kind, "S": _log_int(rng, 1, 16384), "F": _width(rng, 64, 16384), "type": dtype,
                 "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), "train": train}
            fits = c["S"] * c["F"] * (2 if dtype == "f32" else 1) <= MAX_GATE
        else:
            E = _log_int(rng, 2, 256 if kind == "route" else 64)
            c = {"kind": kind, "T": _log_int(rng, 1, 8192), "k": _log_int(rng, 1, min(E, 8)), "E": E}
            S = c["T"] * c["k"]
            if kind == "route":
                c.update(D=_width(rng, 64, 8192), type=dtype, align=rng.choice([1, 128]), drop=rng.random() < 0.3, train=train)
                fits = (S + min(S, E) * (c["align"] - 1)) * c["D"] * (2 if dtype == "f32" else 1) <= MAX_ROUTE
            elif kind == "experts":
                c.update(K=_width(rng, 64, 8192), N=_width(rng, 64, 8192), type=dtype,
                         align=128 if train else rng.choice([1, 128]), train=train)
                fits = ((S + min(S, E) * 64) * c["K"] * c["N"] * (3 if train else 1) <= MAX_LINEAR
                        and E * c["K"] * c["N"] <= MAX_WEIGHTS // (2 if train else 1))
            else:
                c.update(D=_width(rng, 64, 4096), F=_width(rng, 64, 4096), type=rng.choice(["bf16", "bf16", "f16"]),
                         act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]))
                fits = 3 * S * c["D"] * c["F"] <= MAX_LINEAR // 2 and 3 * E * c["D"] * c["F"] <= MAX_WEIGHTS
        if fits:
            return c


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _up(n, to):
    return (n + to - 1) // to * to


def _activations(g, T, D, dtype):
    """Normal values, a few channels much larger than the others."""
    x = torch.randn((T, D), generator=g, device=DEV)
    x *= torch.where(torch.rand((D,), generator=g, device=DEV) < 0.01, 8.0, 1.0)
    return x.to(dtype)


def _room_f8(K, *rows):
    """Room for e4m3 rows of whole blocks, zeros behind their values, and for their scales."""
    q = torch.zeros((*rows, _up(K, BLOCK)), dtype=torch.uint8, device=DEV).view(F8)[..., :K]
    return q, torch.zeros((*rows, _up(_up(K, BLOCK) // BLOCK, 4)), dtype=torch.uint8, device=DEV).view(E8)[..., :_up(K, BLOCK) // BLOCK]


def _weight_f8(g, scales, N, K, *lead):
    """A weight as it is kept between calls: e4m3 with a scale for each 128 x 128 values, powers of two or any."""
    w = torch.randn((*lead, N, K), generator=g, device=DEV) / math.sqrt(K)
    q, s = _room_f8(K, *lead, N)
    if scales == "pow2":
        v, s1 = _plain_weight(w)
        s = s[..., : s1.shape[-2], :]
        s.view(torch.uint8).copy_(_exponent_bytes(s1))
    else:
        b = _tiles(w)
        s = (b.abs().amax((-3, -1)) / 448).clamp(min=1e-30)
        v = _untiled(b / s[..., :, None, :, None], N, K).to(F8).float()
    q.view(torch.uint8).copy_(v.to(F8).view(torch.uint8))
    return q, s


def _routing(g, c):
    """Each token's experts, the most probable of skewed logits, and their weights; with drop some are taken out (-1)."""
    T, k, E = c["T"], c["k"], c["E"]
    logits = torch.randn((T, E), generator=g, device=DEV) + 0.5 * torch.randn((E,), generator=g, device=DEV)
    top, experts = logits.topk(k, 1)
    experts, weights = experts.to(torch.int32), torch.softmax(top, 1)
    if c.get("drop"):
        experts = torch.where(torch.rand((T, k), generator=g, device=DEV) < 0.1, -1, experts)
    return experts, weights


def _capacity(c):
    """Positions that the sorted rows can take, whatever the experts are."""
    n, a = c["T"] * c["k"], c.get("align", 1)
    return (n + min(n, c["E"]) * (a - 1)) // a * a


def _zeros(rows, cols, dtype):
    return torch.zeros((rows, cols), dtype=dtype, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    c, dt = case, TYPES[case["type"]]
    s = {"case": c}
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        s["x"] = _activations(g, M, K, dt)
        s["q"], s["qs"] = _room_f8(K, M)
        s["y"] = _zeros(M, N, dt)
        s["bias"] = 0.1 * torch.randn((N,), generator=g, device=DEV) if c["bias"] else None
        if c["train"]:
            s["w"] = (torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K)).to(dt)
            s["dy"] = (1e-4 * torch.randn((M, N), generator=g, device=DEV)).to(dt)
        else:
            s["w8"], s["ws"] = _weight_f8(g, c["scales"], N, K)
        return s
    if c["kind"] == "gate":
        S, F = c["S"], c["F"]
        s["gu"] = torch.randn((S, 2 * F), generator=g, device=DEV).to(dt)
        if c["train"]:
            s["dh"] = torch.randn((S, F), generator=g, device=DEV).to(dt)
            s["h"], s["dgu"] = _zeros(S, F, dt), _zeros(S, 2 * F, dt)
        else:
            s["q"], s["qs"] = _room_f8(F, S)
        return s
    T, E, S = c["T"], c["E"], _capacity(c)
    s["experts"], s["weights"] = _routing(g, c)
    if c["kind"] == "route":
        D = c["D"]
        s["x"], s["ys"] = _activations(g, T, D, dt), torch.randn((S, D), generator=g, device=DEV).to(dt)
        s["xs"], s["out"] = _zeros(S, D, dt), _zeros(T, D, dt)
        if c["train"]:
            s["dout"], s["dxs"] = (torch.randn((n, D), generator=g, device=DEV).to(dt) for n in (T, S))
            s["dys"], s["dx"] = _zeros(S, D, dt), _zeros(T, D, dt)
    elif c["kind"] == "experts":
        N, K = c["N"], c["K"]
        s["x"] = _activations(g, T, K, dt)
        s["offsets"], s["rows"], s["places"] = _plain_sort(s["experts"], E, c["align"], S)
        s["w8"], s["ws"] = _weight_f8(g, "pow2", N, K, E)
        s["q"], s["qs"] = _room_f8(K, S)
        s["y"] = _zeros(S, N, dt)
        if c["train"]:
            s["wt8"], s["wts"] = _room_f8(N, E, K)
            s["wt8"].view(torch.uint8).copy_(s["w8"].view(torch.uint8).transpose(1, 2))
            s["wts"] = s["wts"][:, : s["ws"].shape[2]]
            s["wts"].view(torch.uint8).copy_(s["ws"].view(torch.uint8).transpose(1, 2))
            s["dy"] = (1e-4 * torch.randn((S, N), generator=g, device=DEV)).to(dt)
            s["dy"][s["rows"] < 0] = 0
            s["dxs"] = _zeros(S, K, dt)
    else:
        D, F = c["D"], c["F"]
        s["x"] = _activations(g, T, D, dt)
        (s["w18"], s["w1s"]), (s["w28"], s["w2s"]) = _weight_f8(g, "pow2", 2 * F, D, E), _weight_f8(g, "pow2", D, F, E)
        (s["q"], s["qs"]), (s["hq"], s["hs"]) = _room_f8(D, S), _room_f8(F, S)
        s["gu"], s["ys"], s["out"] = _zeros(S, 2 * F, dt), _zeros(S, D, dt), _zeros(T, D, dt)
    return s


# ---- the operators in plain form: 32 bits, rounded once at the end -----------------------------------------------------
def _power(p):
    """2^p, exactly."""
    return ((p + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent_bytes(s):
    return (s.view(torch.int32) >> 23).to(torch.uint8)


def _scale(a):
    """The exponent of the smallest power of two times which 448, the largest e4m3 value, is a or more; -100 at least."""
    m, e = torch.frexp(a)
    p = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(a > 0, p, -100).clamp(min=-100)


def _plain_rows(x):
    """(e4m3 values of rows as fp32, scales of their blocks)."""
    rows, K = x.shape
    b = torch.nn.functional.pad(x.float(), (0, _up(K, BLOCK) - K)).reshape(rows, -1, BLOCK)
    p = _scale(b.abs().amax(2))
    return (b * _power(-p)[..., None]).to(F8).float().reshape(rows, -1)[:, :K], _power(p)


def _tiles(w):
    N, K = w.shape[-2:]
    return torch.nn.functional.pad(w.float(), (0, _up(K, BLOCK) - K, 0, _up(N, BLOCK) - N)).reshape(
        *w.shape[:-2], _up(N, BLOCK) // BLOCK, BLOCK, _up(K, BLOCK) // BLOCK, BLOCK)


def _untiled(b, N, K):
    return b.reshape(*b.shape[:-4], b.shape[-4] * BLOCK, b.shape[-2] * BLOCK)[..., :N, :K]


def _plain_weight(w):
    b = _tiles(w)
    p = _scale(b.abs().amax((-3, -1)))
    return _untiled((b * _power(-p)[..., :, None, :, None]).to(F8).float(), *w.shape[-2:]), _power(p)


def _values(q, s):
    """What e4m3 rows with the scales of their blocks stand for."""
    return q.float() * s.float().repeat_interleave(BLOCK, -1)[..., : q.shape[-1]]


def _weight_values(q, s):
    return _values(q, s.float().repeat_interleave(BLOCK, -2)[..., : q.shape[-2], :])


def _plain_sort(experts, E, align, S):
    """offsets of the experts' rows, the slot (token * k + choice) of each position, the position of each slot."""
    flat = experts.reshape(-1).long()
    n = flat.numel()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    counts = torch.zeros((E + 1,), dtype=torch.long, device=DEV).scatter_add_(0, key, torch.ones_like(key))
    order = torch.argsort(key, stable=True)
    ends = torch.cumsum((counts[:E] + align - 1) // align * align, 0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    first = torch.cumsum(counts, 0) - counts
    e = key[order]
    at = torch.where(e < E, offsets[e.clamp(max=E)] + torch.arange(n, device=DEV) - first[e], S)
    rows = torch.where(torch.arange(S + 1, device=DEV) < ends[-1], -1, -2)
    rows[at] = torch.where(e < E, order, -2)
    places = torch.empty_like(flat)
    places[order] = torch.where(e < E, at, -1)
    return offsets.int(), rows[:S].int(), places.reshape(experts.shape).int()


def _plain_gather(x, rows, k, into):
    got = torch.where((rows >= 0)[:, None], x[(rows.long() // k).clamp(min=0)], torch.zeros_like(x[:1]))
    return torch.where((rows >= -1)[:, None], got, into)


def _taken(ys, places):
    """[T, k, D]: the rows of each token's experts, zeros where it has none."""
    return torch.where((places >= 0)[..., None], ys.float()[places.long().clamp(min=0)], 0.0)


def _plain_combine(ys, places, weights, dt):
    t = _taken(ys, places)
    return (t if weights is None else t * weights[..., None]).sum(1).to(dt)


def _plain_combine_backward(s, dt, rows, places):
    k, dout = places.shape[1], s["dout"].float()
    slot = rows.long().clamp(min=0)
    d = (s["weights"].reshape(-1)[slot][:, None] * dout[slot // k]).to(dt)
    d = torch.where((rows >= 0)[:, None], d, torch.zeros_like(d))
    return torch.where((rows >= -1)[:, None], d, s["dys"]), (_taken(s["ys"], places) * dout[:, None]).sum(2)


def _plain_route(s, c, dt):
    offsets, rows, places = _plain_sort(s["experts"], c["E"], c["align"], s["xs"].shape[0])
    got = {"offsets": offsets, "rows": rows, "places": places, "xs": _plain_gather(s["x"], rows, c["k"], s["xs"]),
           "out": _plain_combine(s["ys"], places, s["weights"], dt)}
    if c["train"]:
        got["dys"], got["dweights"] = _plain_combine_backward(s, dt, rows, places)
        got["dx"] = _plain_combine(s["dxs"], places, None, dt)
    return got


def _by_expert(offsets, S):
    """The expert of each position and its place among the expert's rows; positions behind the last: the last expert's."""
    at = torch.arange(S, device=DEV)
    e = (torch.searchsorted(offsets.long(), at, right=True) - 1).clamp(max=offsets.numel() - 2)
    return e, at - offsets.long()[e]


def _spread(v, e, i, E, room, live):
    """Rows [S, D] as [E, room, D], zeros in between."""
    b = torch.zeros((E * room + 1, v.shape[1]), device=DEV)
    b[torch.where(live, e * room + i, E * room)] = v
    return b[:-1].reshape(E, room, -1)


def _plain_expert_product(v, offsets, w, s):
    """Rows [S, K] times their experts' weights [E, N, K]: few rows take copies of them, many are laid out by expert."""
    S, E = v.shape[0], w.shape[0]
    e, i = _by_expert(offsets, S)
    if S <= E:
        return torch.bmm(_weight_values(w[e], s[e]), v[:, :, None])[:, :, 0]
    room, live = int((offsets[1:] - offsets[:-1]).max()), torch.arange(S, device=DEV) < offsets[-1]
    y = torch.bmm(_spread(v, e, i, E, room, live), _weight_values(w, s).transpose(1, 2).contiguous())
    return y.reshape(E * room, -1)[(e * room + i).clamp(max=E * room - 1)]


def _plain_expert_dw(dy, x, offsets, E):
    """For each expert dy^T x over its rows, [E, N, K]."""
    e, i = _by_expert(offsets, dy.shape[0])
    room, live = int((offsets[1:] - offsets[:-1]).max()), torch.arange(dy.shape[0], device=DEV) < offsets[-1]
    return torch.bmm(_spread(dy, e, i, E, room, live).transpose(1, 2).contiguous(), _spread(x, e, i, E, room, live))


def _rows_of(x, rows, k):
    return torch.where((rows >= 0)[:, None], x.float()[(rows.long() // k).clamp(min=0)], 0.0)


def _plain_quantized(x):
    q, s = _plain_rows(x)
    return _values(q, s)


def _plain_linear(s, c, dt):
    x = _plain_quantized(s["x"])
    w = _weight_values(*_plain_weight(s["w"])) if c["train"] else _weight_values(s["w8"], s["ws"])
    y = x @ w.T
    y = (y if s["bias"] is None else y + s["bias"]).to(dt)
    if not c["train"]:
        return y
    dw = _plain_quantized(s["dy"].T) @ _plain_quantized(s["x"].T).T
    return {"y": y, "dx": (_plain_quantized(s["dy"]) @ w).to(dt), "dw": dw}


def _plain_experts(s, c, dt):
    E, rows, offsets = c["E"], s["rows"], s["offsets"]
    x, live = _rows_of(s["x"], rows, c["k"]), (rows >= -1)[:, None]
    y = torch.where(live, _plain_expert_product(_plain_quantized(x), offsets, s["w8"], s["ws"]).to(dt), s["y"])
    if not c["train"]:
        return y
    dxs = _plain_expert_product(_plain_quantized(s["dy"]), offsets, s["wt8"], s["wts"]).to(dt)
    dxs = torch.where(live, dxs, s["dxs"])
    dw = _plain_expert_dw(_plain_quantized(s["dy"].T).T, _plain_quantized(x.T).T, offsets, E)
    return {"y": y, "dx": _plain_combine(dxs, s["places"], None, dt), "dw": dw}


def _plain_act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
    return torch.relu(z)


def _plain_act_slope(z, act):
    if act == "silu":
        t = torch.sigmoid(z)
        return t * (1 + z * (1 - t))
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        t = torch.sigmoid(k * (z + 0.044715 * z * z * z))
        return t + z * t * (1 - t) * k * (1 + 3 * 0.044715 * z * z)
    return (z > 0).to(z.dtype)


def _plain_gated(gu, act):
    g, u = gu.float().chunk(2, 1)
    return _plain_act(g, act) * u


def _plain_gate(s, c, dt):
    h = _plain_gated(s["gu"], c["act"])
    if not c["train"]:
        q, p = _plain_rows(h)
        return {"q": q.to(F8), "scale": _exponent_bytes(p).view(E8)}
    g, u = s["gu"].float().chunk(2, 1)
    dh = s["dh"].float()
    dgu = torch.cat([dh * u * _plain_act_slope(g, c["act"]), dh * _plain_act(g, c["act"])], 1)
    return {"h": h.to(dt), "dgu": dgu.to(dt)}


def _plain_block(s, c, dt):
    """Operator after operator, each rounded at its own end."""
    offsets, rows, places = _plain_sort(s["experts"], c["E"], 1, s["ys"].shape[0])
    x = _plain_quantized(_rows_of(s["x"], rows, c["k"]))
    gu = _plain_expert_product(x, offsets, s["w18"], s["w1s"]).to(dt)
    ys = _plain_expert_product(_plain_quantized(_plain_gated(gu, c["act"])), offsets, s["w28"], s["w2s"]).to(dt)
    return _plain_combine(ys, places, s["weights"], dt)


def run(state):
    s, c = state, state["case"]
    dt = TYPES[c["type"]]
    if own:
        return _run_own(s, c)
    return {"linear": _plain_linear, "route": _plain_route, "experts": _plain_experts, "gate": _plain_gate,
            "block": _plain_block}[c["kind"]](s, c, dt)


# ---- the same through the framework's operators ------------------------------------------------------------------------
def _run_own(s, c):
    from paper_1911_04477_amd import binding as B

    if c["kind"] == "linear":
        B.bnn_quant_blocks_f8(s["x"], s["q"], s["qs"])
        if not c["train"]:
            return B.bnn_linear_f8(s["q"], s["qs"], s["w8"], s["ws"], s["bias"], out=s["y"])
        w, wt = B.bnn_quant_weight_f8(s["w"])
        y = B.bnn_linear_f8(s["q"], s["qs"], *w, s["bias"], out=s["y"])
        dx = B.bnn_linear_f8(*B.bnn_quant_blocks_f8(s["dy"]), *wt, dtype=s["x"].dtype)
        dw = B.bnn_linear_f8(*B.bnn_quant_columns_f8(s["dy"]), *B.bnn_quant_columns_f8(s["x"]), dtype=torch.float32)
        return {"y": y, "dx": dx, "dw": dw}
    if c["kind"] == "gate":
        if not c["train"]:
            q, scale = B.bnn_gated_act_f8(s["gu"], act=c["act"], q=s["q"], scale=s["qs"])
            return {"q": q, "scale": scale}
        h = B.bnn_gated_act(s["gu"], act=c["act"], out=s["h"])
        return {"h": h, "dgu": B.bnn_gated_act_backward(s["gu"], s["dh"], act=c["act"], out=s["dgu"])}
    if c["kind"] == "route":
        offsets, rows, places = B.bnn_expert_sort(s["experts"], c["E"], align=c["align"])
        got = {"offsets": offsets, "rows": rows, "places": places, "xs": B.bnn_expert_gather(s["x"], rows, c["k"], out=s["xs"]),
               "out": B.bnn_expert_combine(s["ys"], places, s["weights"], out=s["out"])}
        if c["train"]:
            got["dys"], got["dweights"] = B.bnn_expert_combine_backward(s["ys"], rows, places, s["weights"], s["dout"],
                                                                        dys=s["dys"])
            got["dx"] = B.bnn_expert_combine(s["dxs"], places, out=s["dx"])
        return got
    if c["kind"] == "experts":
        B.bnn_quant_blocks_f8(s["x"], s["q"], s["qs"], rows=s["rows"], k=c["k"])
        y = B.bnn_expert_linear_f8(s["q"], s["qs"], s["offsets"], s["w8"], s["ws"], out=s["y"])
        if not c["train"]:
            return y
        dxs = B.bnn_expert_linear_f8(*B.bnn_quant_blocks_f8(s["dy"]), s["offsets"], s["wt8"], s["wts"], out=s["dxs"])
        dw = B.bnn_expert_linear_f8_dw(*B.bnn_quant_columns_f8(s["dy"]),
                                       *B.bnn_quant_columns_f8(s["x"], rows=s["rows"], k=c["k"]), s["offsets"])
        return {"y": y, "dx": B.bnn_expert_combine(dxs, s["places"]), "dw": dw}
    offsets, rows, places = B.bnn_expert_sort(s["experts"], c["E"])
    B.bnn_quant_blocks_f8(s["x"], s["q"], s["qs"], rows=rows, k=c["k"])
    B.bnn_expert_linear_f8(s["q"], s["qs"], offsets, s["w18"], s["w1s"], out=s["gu"])
    B.bnn_gated_act_f8(s["gu"], act=c["act"], q=s["hq"], scale=s["hs"])
    B.bnn_expert_linear_f8(s["hq"], s["hs"], offsets, s["w28"], s["w2s"], out=s["ys"])
    return B.bnn_expert_combine(s["ys"], places, s["weights"], out=s["out"])


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    c, size = case, TYPES[case["type"]].itemsize
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        if c["train"]:
            return {"bytes": (2 * M * K + 2 * M * N + N * K) * size + 4 * N * K, "flops": 6 * M * N * K}
        return {"bytes": M * K * size + N * K + M * N * size + (4 * N if c["bias"] else 0), "flops": 2 * M * N * K}
    if c["kind"] == "gate":
        n = c["S"] * c["F"]
        return {"bytes": n * size * (3 + 3) if c["train"] else n * (2 * size + 1), "flops": n * (40 if c["train"] else 12)}
    T, n = c["T"], c["T"] * c["k"]
    used = c["E"] * (1 - (1 - 1 / c["E"]) ** n)  # experts with rows of their own, where they are equally likely
    if c["kind"] == "route":
        D = c["D"]
        plan = 4 * (3 * n + c["E"]) + 4 * n
        if c["train"]:  # x, ys, dxs in, xs, out, dx out; dout in, dys and the weights' gradients out
            return {"bytes": plan + 4 * n + (4 * n + 4 * T) * D * size, "flops": 5 * n * D}
        return {"bytes": plan + 2 * (n + T) * D * size, "flops": 2 * n * D}
    if c["kind"] == "experts":
        N, K = c["N"], c["K"]
        if c["train"]:
            return {"bytes": (2 * T * K + 2 * n * N) * size + 2 * used * N * K + 4 * c["E"] * N * K, "flops": 6 * n * N * K}
        return {"bytes": (T * K + n * N) * size + used * N * K, "flops": 2 * n * N * K}
    D, F = c["D"], c["F"]
    return {"bytes": 2 * T * D * size + 8 * n + 3 * used * D * F, "flops": 6 * n * D * F}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
class _Exact:
    """Each operator from its formula, values and sums in 64 bits, experts one after the other."""

    @staticmethod
    def two(p):
        """2^p from its bits."""
        return ((p.long() + 1023) << 52).view(torch.float64)

    @staticmethod
    def exponent(top):
        """The least whole p with top <= 448 * 2^p, at least -100."""
        m, e = torch.frexp(top / 448.0)
        p = torch.where(m == 0.5, e - 1, e)
        return torch.where(top > 0, p, torch.full_like(p, -100)).clamp(min=-100)

    def e4m3(self, v):
        """The nearest value with three bits behind the leading one, ties to even, steps of 2^-9 at the lower end."""
        _, e = torch.frexp(v)
        step = self.two((e - 1).clamp(min=-6) - 3)
        return torch.round(v / step) * step

    def blocks(self, x):
        """Rows as the values that their 8-bit form stands for, in blocks of 128."""
        x = x.double()
        got = torch.empty_like(x)
        for lo in range(0, x.shape[1], BLOCK):
            part = x[:, lo: lo + BLOCK]
            unit = self.two(self.exponent(part.abs().max(dim=1, keepdim=True).values))
            got[:, lo: lo + BLOCK] = self.e4m3(part / unit) * unit
        return got

    def weight(self, w):
        w = w.double()
        got = torch.empty_like(w)
        for n in range(0, w.shape[0], BLOCK):
            band = w[n: n + BLOCK]
            for lo in range(0, w.shape[1], BLOCK):
                part = band[:, lo: lo + BLOCK]
                unit = self.two(self.exponent(part.abs().max()))
                got[n: n + BLOCK, lo: lo + BLOCK] = self.e4m3(part / unit) * unit
        return got

    @staticmethod
    def stored(q, s):
        """What a stored weight stands for."""
        n = torch.arange(q.shape[0], device=DEV) // BLOCK
        k = torch.arange(q.shape[1], device=DEV) // BLOCK
        return q.double() * s.double()[n][:, k]

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

    def gated(self, gu, name):
        F = gu.shape[1] // 2
        return self.act(gu[:, :F].double(), name)[0] * gu[:, F:].double()

    @staticmethod
    def slots(experts, E, align):
        """Expert by expert its first position, the slots that chose it and the end of its padded rows."""
        flat, at, got = experts.reshape(-1).cpu(), 0, []
        for e in range(E):
            chose = torch.nonzero(flat == e)[:, 0].to(DEV)
            end = at + -(-chose.numel() // align) * align
            got.append((at, chose, end))
            at = end
        return got

    def route(self, s, c):
        k, D, S = c["k"], c["D"], s["xs"].shape[0]
        T = c["T"]
        w = s["weights"].double().reshape(-1)
        got = {"xs": torch.zeros((S, D), dtype=torch.float64, device=DEV), "out": torch.zeros((T, D), dtype=torch.float64, device=DEV)}
        if c["train"]:
            got.update(dys=torch.zeros_like(got["xs"]), dx=torch.zeros_like(got["out"]), dweights=torch.zeros_like(w))
        for at, slot, _ in self.slots(s["experts"], c["E"], c["align"]):
            here, token = slice(at, at + slot.numel()), slot // k
            got["xs"][here] = s["x"][token].double()
            got["out"].index_add_(0, token, s["ys"][here].double() * w[slot, None])
            if c["train"]:
                d = s["dout"][token].double()
                got["dys"][here] = d * w[slot, None]
                got["dweights"][slot] = (d * s["ys"][here].double()).sum(dim=1)
                got["dx"].index_add_(0, token, s["dxs"][here].double())
        if c["train"]:
            got["dweights"] = got["dweights"].reshape(T, k)
        return got

    def experts(self, s, c):
        k, S, N, K, E = c["k"], s["y"].shape[0], c["N"], c["K"], c["E"]
        x8 = self.blocks(s["x"])
        y = torch.zeros((S, N), dtype=torch.float64, device=DEV)
        if c["train"]:
            dx = torch.zeros((c["T"], K), dtype=torch.float64, device=DEV)
            dw = torch.zeros((E, N, K), dtype=torch.float64, device=DEV)
            dt = TYPES[c["type"]]
        for e, (at, slot, end) in enumerate(self.slots(s["experts"], E, c["align"])):
            if not slot.numel():
                continue
            here, w = slice(at, at + slot.numel()), self.stored(s["w8"][e], s["ws"][e])
            y[here] = torch.mm(x8[slot // k], w.t())
            if c["train"]:
                dy = s["dy"][here]
                dx.index_add_(0, slot // k, torch.mm(self.blocks(dy), w).to(dt).double())
                dw[e] = torch.mm(self.blocks(dy.t()), self.blocks(s["x"][slot // k].t()).t())
        return {"y": y, "dx": dx, "dw": dw} if c["train"] else y

    def block(self, s, c, dt):
        """The layer's definition has the two products' results in the tensors' type."""
        x8, out = self.blocks(s["x"]), torch.zeros((c["T"], c["D"]), dtype=torch.float64, device=DEV)
        w = s["weights"].double().reshape(-1)
        for e, (at, slot, _) in enumerate(self.slots(s["experts"], c["E"], 1)):
            if not slot.numel():
                continue
            gu = torch.mm(x8[slot // c["k"]], self.stored(s["w18"][e], s["w1s"][e]).t()).to(dt)
            y = torch.mm(self.blocks(self.gated(gu, c["act"])), self.stored(s["w28"][e], s["w2s"][e]).t()).to(dt)
            out.index_add_(0, slot // c["k"], y.double() * w[slot, None])
        return out


def exact(case, seed):
    s, c, E = prepare(case, seed), case, _Exact()
    if c["kind"] == "linear":
        x = E.blocks(s["x"])
        w = E.weight(s["w"]) if c["train"] else E.stored(s["w8"], s["ws"])
        y = torch.mm(x, w.t())
        y = y if s["bias"] is None else y + s["bias"].double()
        if not c["train"]:
            return y
        return {"y": y, "dx": torch.mm(E.blocks(s["dy"]), w), "dw": torch.mm(E.blocks(s["dy"].t()), E.blocks(s["x"].t()).t())}
    if c["kind"] == "gate":
        if not c["train"]:
            h = E.gated(s["gu"], c["act"])
            q, p = torch.zeros_like(h), []
            for lo in range(0, h.shape[1], BLOCK):
                part = h[:, lo: lo + BLOCK]
                p.append(E.exponent(part.abs().max(dim=1, keepdim=True).values))
                q[:, lo: lo + BLOCK] = E.e4m3(part / E.two(p[-1]))
            return {"q": q, "scale": E.two(torch.cat(p, 1))}
        a, slope = E.act(s["gu"][:, : c["F"]].double(), c["act"])
        u, dh = s["gu"][:, c["F"]:].double(), s["dh"].double()
        return {"h": a * u, "dgu": torch.cat([dh * u * slope, dh * a], 1)}
    if c["kind"] == "route":
        return E.route(s, c)
    return E.experts(s, c) if c["kind"] == "experts" else E.block(s, c, TYPES[c["type"]])
