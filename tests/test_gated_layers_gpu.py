"""The 8-bit linear layer, the gated norms and the gated feed-forward block against their formulas in 64 bits.

Tolerances are bounds from the roundings of each operator: u is the unit roundoff of the type that a value is rounded to
(2^-8 bf16, 2^-11 fp16, 2^-24 fp32), a sum of n fp32 terms is off by at most n u times the sum of their magnitudes."""
import itertools
import math

import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U32 = U[torch.float32]
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}  # spacing of the smallest numbers
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-6


def gen(*key):
    g = torch.Generator(device=DEV)
    g.manual_seed(hash(key) % (1 << 31))
    return g


def normal(g, *shape, std=1.0):
    return std * torch.randn(shape, generator=g, device=DEV)


def strided(t, gap):
    """The same values in rows that are `gap` elements longer; what lies between them must not be read into a result."""
    if gap == 0:
        return t
    filler = -1 if not t.dtype.is_floating_point else float("nan")
    big = torch.full((t.shape[0], t.shape[1] + gap), filler, dtype=t.dtype, device=t.device)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def close(got, want, bound, name=""):
    """Elementwise |got - want| <= bound, where bound already holds every rounding."""
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / bound).nan_to_num(1e9).max()):.3g} of the bound, "
                                 f"first at {bad.nonzero()[0].tolist()}: {float(got.double()[tuple(bad.nonzero()[0])])} for {float(want[tuple(bad.nonzero()[0])])}")


def rounded(want, dtype):
    return U[dtype] * want.abs() + TINY[dtype]


# ---------------------------------------------------------------- quantizer
def quant_ref(x):
    """The definition, operation by operation in fp32."""
    x = x.float()
    a = x.abs().amax(1)
    a = torch.where(x.isnan().any(1), torch.full_like(a, float("nan")), a)
    zero = a < 2.0 ** -100
    full = torch.full_like(a, 127.0)
    scale = torch.where(zero, torch.zeros_like(a), a / full)
    scale = torch.where(a.isfinite(), scale, a)
    inv = torch.where(zero | ~a.isfinite(), torch.zeros_like(a), full / a)
    q = (x * inv[:, None]).round()
    return torch.where(inv[:, None] == 0, torch.zeros_like(q), q).to(torch.int8), scale


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,K,gap", [(1, 1, 0), (5, 7, 0), (3, 8, 3), (9, 9, 0), (4, 511, 1), (2, 512, 0), (6, 513, 2), (7, 2048, 0),
                                        (2, 2051, 0), (3, 8191, 5), (2, 8192, 0), (2, 8195, 0), (1, 32768, 0), (2, 32771, 1),
                                        (1, 70001, 0)])
def test_quant_rows(rows, K, gap, dtype):
    print(f"quant {rows} x {K} gap {gap} {dtype}", flush=True)
    x = normal(gen(rows, K, gap), rows, K).to(dtype)
    room = torch.full((rows, K + gap + 3), 77, dtype=torch.int8, device=DEV)
    scale = torch.full((rows,), -1.0, device=DEV)
    B.bnn_quant_rows_i8(strided(x, gap), room[:, :K], scale)
    q, s = quant_ref(x)
    assert torch.equal(room[:, :K], q) and torch.equal(scale, s)
    assert bool((room[:, K:] == 77).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_quant_rows_of_special_values(dtype):
    x = normal(gen(1), 12, 300).to(dtype)
    x[0] = 0
    x[1, 7] = float("inf")
    x[2, 299] = float("nan")
    x[3, 0], x[3, 1] = float("-inf"), float("nan")
    x[4] = 2.0 ** -130 if dtype != F16 else 0.0  # below 2^-100: zero
    x[5] = TINY[dtype]
    x[6] = torch.finfo(dtype).max
    x[7] = -torch.finfo(dtype).max
    x[8] = -0.0
    x[9] = torch.arange(300, device=DEV) / 2 - 63.5  # halves: ties to even
    x[9, 200:] = 127.0
    x[10, 1:] = 0
    q, s = B.bnn_quant_rows_i8(x)
    rq, rs = quant_ref(x)
    assert torch.equal(q, rq) and torch.equal(s.nan_to_num(-5.0), rs.nan_to_num(-5.0)) and torch.equal(s.isnan(), rs.isnan())
    assert s[0] == 0 and s[1] == float("inf") and s[2].isnan() and s[3].isnan() and s[8] == 0
    w, ws = B.bnn_quant_rows_i8(normal(gen(2), 40, 300))
    y = B.bnn_linear_i8(q, s, w, ws, dtype=F32)
    assert bool(y[1:4].isnan().all()) and bool((y[0] == 0).all()) and bool(y[[4, 5, 8, 9, 10, 11]].isfinite().all())  # 6, 7: past fp32


# ---------------------------------------------------------------- int8 linear layer
LINEAR = [(1, 1, 1), (1, 17, 5), (3, 64, 64), (16, 16, 256), (16, 40, 2321), (17, 33, 100), (64, 65, 129), (50, 1000, 3000), (65, 130, 127),
          (128, 128, 128), (129, 257, 384), (256, 512, 1000), (300, 520, 2064), (513, 1030, 641), (4101, 4105, 144), (2000, 16400, 300),
          (600, 3000, 400), (1000, 4500, 272), (1, 4096, 4096)]


def linear_ref(a, sa, b, sb, bias):
    y = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    return y if bias is None else y + bias.double()


@pytest.mark.parametrize("dtype,with_bias,gap", [(BF16, False, 0), (F16, True, 16), (F32, True, 3)])
@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear_i8(M, N, K, dtype, with_bias, gap):
    print(f"linear {M} x {N} x {K} {dtype} gap {gap}", flush=True)
    g = gen(M, N, K)
    a = torch.randint(-128, 128, (M, K), generator=g, device=DEV, dtype=torch.int8)
    b = torch.randint(-128, 128, (N, K), generator=g, device=DEV, dtype=torch.int8)
    # rows in 16-byte strides (gap 0), in such strides with other values between, or at any address
    a_, b_ = (strided(t, gap if gap % 16 else (-K) % 16 + gap) for t in (a, b))
    sa = torch.rand((M,), generator=g, device=DEV) / (100 * math.sqrt(K)) + 1e-5
    sb = torch.rand((N,), generator=g, device=DEV) / 50 + 1e-5
    bias = normal(g, N) if with_bias else None
    out = torch.full((M, N + gap), -3.0, dtype=dtype, device=DEV)
    y = B.bnn_linear_i8(a_, sa, b_, sb, bias, out=out[:, :N])
    want = linear_ref(a, sa, b, sb, bias)
    product = want if bias is None else want - bias.double()
    close(y, want, rounded(want, dtype) + 4 * U32 * (product.abs() + (0 if bias is None else bias.double().abs())), "y")
    assert bool((out[:, N:] == -3.0).all())


def test_linear_i8_largest_sums():
    """Sums next to the ends of 32 bits."""
    K = 131071
    a = torch.full((18, K), -128, dtype=torch.int8, device=DEV)
    b = torch.full((3, K), -128, dtype=torch.int8, device=DEV)
    b[1] = 127
    b[2, ::2] = 127
    one = torch.ones((18,), device=DEV)
    for M in (2, 18):
        y = B.bnn_linear_i8(a[:M], one[:M], b, one[:3], dtype=F32)
        assert torch.equal(y.double(), (a[:M].double() @ b.double().t()).float().double())


def test_linear_i8_offsets_beyond_32_bits():
    """Rows past 2^32 bytes of either operand and of the output."""
    K, stride = 64, 1 << 20
    big = torch.zeros((4300, stride), dtype=torch.int8, device=DEV)  # 4.5 GB
    g = gen(7)
    small = torch.randint(-128, 128, (4300, K), generator=g, device=DEV, dtype=torch.int8)
    big[:, :K] = small
    other = torch.randint(-128, 128, (70, K), generator=g, device=DEV, dtype=torch.int8)
    one = torch.ones((4300,), device=DEV)
    want = (small.double() @ other.double().t()).float()
    assert torch.equal(B.bnn_linear_i8(big[:, :K], one, other, one[:70], dtype=F32), want)
    assert torch.equal(B.bnn_linear_i8(other, one[:70], big[:, :K], one, dtype=F32), want.t())
    assert torch.equal(B.bnn_linear_i8(other[:3], one[:3], big[:, :K], one, dtype=F32), want.t()[:3])
    out = big.view(torch.float32)[:, :70]  # the rows of the output a megabyte apart
    B.bnn_linear_i8(small, one, other, one[:70], out=out)
    assert torch.equal(out, want)


# ---------------------------------------------------------------- norms
def norm_inputs(g, rows, D, dtype, rtype, post, pre, gate, vectors):
    s = {"gate_rows": {"none": 1, "channel": max(rows, 1), "token": 1}.get(gate, gate if isinstance(gate, int) else 1), "gate": None}
    groups = -(-rows // s["gate_rows"])
    if gate != "none":
        s["gate"] = normal(g, groups, D).to(dtype)
    on = {"res_scale": vectors, "w_post": vectors and post != "none", "bias_post": vectors and post == "layer",
          "w_pre": vectors and pre != "none", "bias_pre": vectors and pre == "layer"}
    for k, v in on.items():
        s[k] = normal(g, D) + (1 if k.startswith("w") else 0) if v else None
    s.update(post=post, pre=pre, eps=EPS)
    b = (normal(g, rows, D) + 0.5).to(dtype)
    r = (2 * normal(g, rows, D) - 0.25).to(rtype)
    return b, r, s


def unit_ref(x, norm):
    if norm == "none":
        return x, torch.ones_like(x[:, :1])
    if norm == "layer":
        x = x - x.mean(1, keepdim=True)
    rs = 1 / ((x * x).mean(1, keepdim=True) + EPS).sqrt()
    return x * rs, rs


def d(t, other):
    return other if t is None else t.double()


def norm_parts(b, r, s):
    one = torch.ones((b.shape[1],), dtype=torch.float64, device=DEV)
    gate = one[None] if s["gate"] is None else s["gate"].double().repeat_interleave(s["gate_rows"], 0)[:b.shape[0]]
    m = d(s["res_scale"], one) * gate
    ub, rsb = unit_ref(b.double(), s["post"])
    p = ub * d(s["w_post"], one) + d(s["bias_post"], 0 * one)
    r1 = r.double() + m * p
    ur, rsr = unit_ref(r1, s["pre"])
    n = ur * d(s["w_pre"], one) + d(s["bias_pre"], 0 * one)
    return {"one": one, "gate": gate, "m": m, "ub": ub, "rsb": rsb, "p": p, "r1": r1, "ur": ur, "rsr": rsr, "n": n}


def norm_bounds(b, r, s, x):
    """A row sum of D values goes through at most 16 + 6 + 16 additions (values of a thread, lanes, waves): a mean or a mean
    square is off by 40 u of the mean magnitude or square, the factor of a row by half that and 3 u, a normed value
    by 64 u of itself and of the row's mean magnitude, which also bounds what the stream's own error does to its norm."""
    reach = 64 * U32
    level = b.double().abs().mean(1, keepdim=True) * x["rsb"] if s["post"] == "layer" else 0.0
    dp = reach * (d(s["w_post"], x["one"]).abs() * (x["ub"].abs() + level) + x["p"].abs())
    dr1 = x["m"].abs() * dp + 4 * U32 * (r.double().abs() + (x["m"] * x["p"]).abs())
    level = x["r1"].abs().mean(1, keepdim=True) * x["rsr"] if s["pre"] == "layer" else 0.0
    from_r = x["rsr"] * (dr1 + (dr1.mean(1, keepdim=True) if s["pre"] == "layer" else 0.0)
                         + x["ur"].abs() * (dr1 * x["ur"].abs()).mean(1, keepdim=True))
    dn = d(s["w_pre"], x["one"]).abs() * (reach * (x["ur"].abs() + level) + 2 * from_r) + reach * x["n"].abs()
    return dr1, dn, from_r


NORM_D = [1, 2, 7, 8, 9, 64, 511, 513, 2047, 2321, 4096, 4097, 8192, 8200, 16384]
NORM_KINDS = [("rms", "rms", "channel", True, BF16, BF16), ("layer", "layer", 3, True, F16, F32), ("none", "rms", "none", False, F32, F32),
              ("rms", "layer", "token", True, BF16, F32), ("layer", "none", "none", True, F16, F16), ("rms", "rms", "none", False, F32, F32)]


@pytest.mark.parametrize("post,pre,gate,vectors,dtype,rtype", NORM_KINDS)
@pytest.mark.parametrize("D", NORM_D)
def test_norm_gate(D, post, pre, gate, vectors, dtype, rtype):
    for rows, gap in ((1, 0), (37, 3)):
        print(f"norm {rows} x {D} {post} {pre} {gate} {dtype} {rtype}", flush=True)
        b, r, s = norm_inputs(gen(rows, D, post, pre), rows, D, dtype, rtype, post, pre, gate, vectors)
        x = norm_parts(b, r, s)
        dr1, dn, _ = norm_bounds(b, r, s, x)
        room = torch.full((rows, D + gap), 5.0, dtype=dtype, device=DEV)
        n_room = room[:, :D] if pre != "none" else None
        r1, n = B.bnn_norm_gate(strided(b, gap), strided(r, gap), n_out=n_room, **s)
        close(r1, x["r1"], rounded(x["r1"], rtype) + dr1, "r'")
        if pre == "none":
            assert n is None
            continue
        close(n, x["n"], rounded(x["n"], dtype) + dn, "n")
        assert bool((room[:, D:] == 5.0).all())
        # 8-bit output: within the rounding to a step of what the fp32 values are, the scale from their largest
        q, qs = torch.full((rows, D + 5), 9, dtype=torch.int8, device=DEV), torch.empty((rows,), device=DEV)
        stream = strided(r, gap).clone()
        again, none = B.bnn_norm_gate(b, stream, q_out=q[:, :D], q_scale=qs, r_out=stream, **s)  # r' in place of r
        assert none is None and torch.equal(again, r1) and bool((q[:, D:] == 9).all())
        top = x["n"].abs().amax(1)
        worst = dn.amax(1)
        assert bool(((qs.double() - top / 127).abs() <= worst / 127 + 2 * U32 * top / 127 + TINY[F32]).all())
        step = qs.double()[:, None]
        close(q[:, :D].double() * step, x["n"], 0.5 * step + dn + worst[:, None] + 4 * U32 * top[:, None], "q")


def test_norm_gate_before_the_first_block():
    r = normal(gen(3), 5, 300).to(BF16)
    w = normal(gen(4), 300)
    r1, n = B.bnn_norm_gate(None, r, post="none", w_pre=w)
    assert r1 is None
    want = unit_ref(r.double(), "rms")[0] * w.double()
    close(n, want, rounded(want, BF16) + 64 * U32 * want.abs(), "n")


def test_norm_gate_keeps_infinities_and_nans_in_their_rows():
    b, r, s = norm_inputs(gen(9), 6, 700, BF16, BF16, "rms", "rms", "channel", True)
    clean = B.bnn_norm_gate(b, r, **s)
    b[1, 3], r[2, 699], b[4] = float("nan"), float("inf"), 0.0
    r1, n = B.bnn_norm_gate(b, r, **s)
    for i in (0, 3, 5):
        assert torch.equal(r1[i], clean[0][i]) and torch.equal(n[i], clean[1][i])
    assert bool(r1[1].isnan().all()) and bool(n[1].isnan().all()) and bool(n[2].isnan().any()) and torch.equal(r1[4], r[4])
    q, qs = B.rows_i8(6, 700, DEV), torch.empty((6,), device=DEV)
    B.bnn_norm_gate(b, r, q_out=q, q_scale=qs, **s)
    assert qs[1].isnan() and qs[2].isnan() and bool((q[1:3] == 0).all()) and bool(qs[[0, 3, 4, 5]].isfinite().all())


def unit_back_ref(e, u, rs, norm):
    if norm == "none":
        return e
    level = e.mean(1, keepdim=True) if norm == "layer" else 0.0
    return rs * (e - level - u * (e * u).mean(1, keepdim=True))


def norm_back_ref(b, r, s, dn, dro):
    x = norm_parts(b, r, s)
    dr = dro + unit_back_ref(dn * d(s["w_pre"], x["one"]), x["ur"], x["rsr"], s["pre"])
    dp = dr * x["m"]
    got = {"dr": dr, "db": unit_back_ref(dp * d(s["w_post"], x["one"]), x["ub"], x["rsb"], s["post"])}
    terms = {"dw_pre": dn * x["ur"], "dbias_pre": dn, "dw_post": dp * x["ub"], "dbias_post": dp, "dres_scale": dr * x["gate"] * x["p"]}
    got.update({k: v.sum(0) for k, v in terms.items() if s[k[1:]] is not None})
    size = {k: v.abs().sum(0) for k, v in terms.items()}
    if s["gate"] is not None:
        at = torch.arange(b.shape[0], device=DEV) // s["gate_rows"]
        t = dr * d(s["res_scale"], x["one"]) * x["p"]
        zero = torch.zeros(s["gate"].shape, dtype=torch.float64, device=DEV)
        got["dgate"], size["dgate"] = zero.index_add(0, at, t), zero.index_add(0, at, t.abs())
    return got, size, x


@pytest.mark.parametrize("post,pre,gate,vectors,dtype,rtype", NORM_KINDS)
@pytest.mark.parametrize("rows,D", [(1, 1), (1, 4096), (2, 9), (37, 64), (5000, 40), (2100, 513), (700, 2321), (1300, 300), (40, 4097), (9, 8200)])
def test_norm_gate_backward(rows, D, post, pre, gate, vectors, dtype, rtype):
    """In fp32 the chain loses at most a few hundred u of a row's own magnitudes; a 16-bit result adds its rounding."""
    print(f"norm backward {rows} x {D} {post} {pre} {gate} {dtype} {rtype}", flush=True)
    g = gen(rows, D, post, pre, 1)
    b, r, s = norm_inputs(g, rows, D, dtype, rtype, post, pre, gate, vectors)
    dn = normal(g, rows, D).to(dtype) if pre != "none" else None
    dro = normal(g, rows, D).to(rtype)
    gap = 3 if rows > 1 else 0
    got = B.bnn_norm_gate_backward(strided(b, gap), strided(r, gap), None if dn is None else strided(dn, gap), strided(dro, gap), **s)
    want, size, x = norm_back_ref(b, r, s, 0.0 * dro.double() if dn is None else dn.double(), dro.double())
    assert set(got) == set(want)

    def row_bound(e, u, rs, norm):  # of the gradient through one norm: magnitudes of its three terms, 256 u of them
        if norm == "none":
            return 256 * U32 * e.abs()
        return 256 * U32 * rs * (e.abs() + e.abs().mean(1, keepdim=True) + (u.abs() + 1) * (e * u).abs().mean(1, keepdim=True)) * (
            1 + (x["r1"].abs().mean(1, keepdim=True) * x["rsr"] if norm == "layer" else 0.0))

    e = 0.0 if dn is None else dn.double() * d(s["w_pre"], x["one"])
    bound_r = 8 * U32 * want["dr"].abs() + (0.0 if dn is None else row_bound(e, x["ur"], x["rsr"], pre)) + 4 * U32 * dro.double().abs()
    close(got["dr"], want["dr"], rounded(want["dr"], rtype) + bound_r, "dr")
    dp = want["dr"] * x["m"]
    e, de = dp * d(s["w_post"], x["one"]), bound_r * (x["m"] * d(s["w_post"], x["one"])).abs()
    back = de if post == "none" else x["rsb"] * (de + de.mean(1, keepdim=True) + x["ub"].abs() * (de * x["ub"].abs()).mean(1, keepdim=True))
    close(got["db"], want["db"], rounded(want["db"], dtype) + back + row_bound(e, x["ub"], x["rsb"], post), "db")
    scale = {"dw_pre": 1.0, "dbias_pre": 1.0}
    for name in set(want) - {"dr", "db"}:
        # terms by 512 u each (they come from the rows' chain), their sum over rows in fp32 by its length at most
        loss = 512 * U32 * size[name] + min(rows, 2100) * U32 * size[name] * scale.get(name, 1.0)
        spill = (0.0 if dn is None else (dn.double().abs() * 2 * norm_bounds(b, r, s, x)[2]).sum(0)) if name == "dw_pre" else (bound_r * (x["m"].abs() + x["gate"].abs()) * (1 + x["p"].abs() + x["ub"].abs())).sum(0) if name not in scale else 0.0  # r' next to zero is off by u of r
        if name == "dgate":
            at = torch.arange(rows, device=DEV) // s["gate_rows"]
            spill = torch.zeros_like(want[name]).index_add(0, at, bound_r * d(s["res_scale"], x["one"]).abs() * x["p"].abs())
        close(got[name], want[name], rounded(want[name], got[name].dtype) + loss + spill, name)
    again = B.bnn_norm_gate_backward(b, r, dn, dro, **s)
    for name in got:
        assert torch.equal(got[name], again[name]), name  # the same sums in the same order


@pytest.mark.parametrize("post,pre,gate", [("rms", "layer", 4), ("layer", "rms", "channel"), ("none", "rms", "token")])
def test_norm_gate_backward_by_differences(post, pre, gate):
    """<gradient, step> against the change of sum(dn * n + dr_out * r') along the step, both halves by the kernels in fp32:
    central differences at h = 2^-6 of a unit step are off by O(h^2) of the third derivatives, within 1 %."""
    g = gen(post, pre)
    rows, D, h = 23, 130, 2.0 ** -6
    b, r, s = norm_inputs(g, rows, D, F32, F32, post, pre, gate, True)
    dn, dro = normal(g, rows, D), normal(g, rows, D)
    grad = B.bnn_norm_gate_backward(b, r, dn, dro, **s)

    def loss(b, r, s):
        r1, n = B.bnn_norm_gate(b, r, **s)
        return float((dn.double() * n.double()).sum() + (dro.double() * r1.double()).sum())

    for name in grad:
        key = name[1:]
        at = {"b": b, "r": r}.get(key, s.get(key))
        step = grad[name] / grad[name].norm() + 0.3 * torch.nn.functional.normalize(normal(g, *at.shape).reshape(1, -1)).reshape(at.shape)
        ends = []
        for sign in (1, -1):
            moved = at + sign * h * step
            ends.append(loss(moved if key == "b" else b, moved if key == "r" else r, s if key in ("b", "r") else {**s, key: moved}))
        want = float((grad[name].double() * step.double()).sum())
        assert abs((ends[0] - ends[1]) / (2 * h) - want) <= 0.01 * abs(want) + 1e-3, name


def test_norm_gate_backward_parts():
    """Missing gradients are zero, unwanted sums are left out, no rows give sums of zero."""
    b, r, s = norm_inputs(gen(5), 30, 200, BF16, F32, "rms", "rms", "channel", True)
    dn, dro = normal(gen(6), 30, 200).to(BF16), normal(gen(7), 30, 200)
    zero = torch.zeros_like
    for x, y in (((dn, None), (dn, zero(dro))), ((None, dro), (zero(dn), dro))):
        one, two = (B.bnn_norm_gate_backward(b, r, *p, **s) for p in (x, y))
        assert all(torch.equal(one[k], two[k]) for k in one)
    first = B.bnn_norm_gate_backward(None, r, dn=dro, dr_out=dro, post="none", w_pre=s["w_pre"])
    assert set(first) == {"dr", "dw_pre"}
    empty = B.bnn_norm_gate_backward(b[:0], r[:0], dn[:0], dro[:0], **{**s, "gate": s["gate"][:0]})
    assert empty["dr"].shape == (0, 200) and all(bool((empty[k] == 0).all()) for k in ("dres_scale", "dw_post", "dw_pre"))


# ---------------------------------------------------------------- gated feed-forward
def act_ref(z, act):
    if act == "silu":
        t = torch.sigmoid(z)
        return z * t, t * (1 + z * (1 - t))
    if act == "gelu":
        t = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * t, t + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k, c = math.sqrt(2 / math.pi), 0.044715
        t = torch.tanh(k * (z + c * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * c * z * z)
    return z.clamp(min=0), (z > 0).double()


GATED = [(1, 1, 1), (1, 40, 17), (3, 200, 64), (16, 64, 33), (17, 65, 130), (64, 520, 100), (65, 127, 129), (128, 128, 256), (200, 1000, 321),
         (257, 257, 513), (1030, 72, 2100), (600, 72, 1500), (4100, 64, 2321)]


def gated_inputs(T, D, F, dtype):
    g = gen(T, D, F)
    return (normal(g, T, D).to(dtype), normal(g, F, D, std=D ** -0.5).to(dtype), normal(g, F, D, std=D ** -0.5).to(dtype),
            normal(g, T, F).to(dtype))


def gated_bounds(x, wg, wu, act, g, u):
    """The fp32 sums by their length, the activation's slope at most 1.13, its evaluation 16 u of |z| + |act|."""
    D = x.shape[1]
    off_g, off_u = ((D + 8) * U32 * (x.double().abs() @ w.double().abs().t()) for w in (wg, wu))
    a, slope = act_ref(g, act)
    off_a = 1.2 * off_g + 16 * U32 * (g.abs() + a.abs())
    return off_g, off_u, off_a, a, slope


@pytest.mark.parametrize("dtype,act,gap", [(BF16, "silu", 0), (F16, "gelu", 8), (BF16, "gelu_tanh", 3), (F16, "relu", 0)])
@pytest.mark.parametrize("T,D,F", GATED)
def test_gated_ff(T, D, F, dtype, act, gap):
    print(f"gated {T} x {D} x {F} {dtype} {act} gap {gap}", flush=True)
    x, wg, wu, _ = gated_inputs(T, D, F, dtype)
    room = torch.full((T, F + gap), 3.0, dtype=dtype, device=DEV)
    saved = B.gated_ff_saved(T, F, DEV)
    h = B.bnn_gated_ff(strided(x, gap), strided(wg, gap), strided(wu, gap), act, out=room[:, :F], saved=saved)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    off_g, off_u, off_a, a, slope = gated_bounds(x, wg, wu, act, g, u)
    want = a * u
    off = off_a * u.abs() + a.abs() * off_u + 4 * U32 * want.abs()
    close(h, want, rounded(want, dtype) + off, "h")
    assert bool((room[:, F:] == 3.0).all())
    assert torch.equal(B.bnn_gated_ff(strided(x, gap), strided(wg, gap), strided(wu, gap), act), h)  # without saving
    close(saved[1], a, off_a + TINY[F32], "act(g)")
    if act != "relu":  # its slope jumps; second derivatives of the others are at most 0.8
        close(saved[0], slope * u, slope.abs() * off_u + (0.9 * off_g + 16 * U32 * (1 + g.abs())) * u.abs() + TINY[F32], "act'(g) u")


@pytest.mark.parametrize("dtype,act,gap", [(BF16, "silu", 0), (F16, "gelu", 3), (BF16, "relu", 8)])
@pytest.mark.parametrize("T,D,F", GATED)
def test_gated_ff_backward(T, D, F, dtype, act, gap):
    """From given saved values: the gradients of both projections are rounded once (u each), then summed in fp32."""
    print(f"gated backward {T} x {D} x {F} {dtype} {act} gap {gap}", flush=True)
    x, wg, wu, dh = gated_inputs(T, D, F, dtype)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    a, slope = act_ref(g, act)
    saved = torch.stack([(slope * u).float(), a.float()])
    dx, dwg, dwu = B.bnn_gated_ff_backward(strided(x, gap), strided(wg, gap), strided(wu, gap), saved, strided(dh, gap))
    dg, du = dh.double() * saved[0].double(), dh.double() * saved[1].double()
    mag = {}
    for name, got, want, size, n in (
            ("dx", dx, dg @ wg.double() + du @ wu.double(), dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs(), 2 * F),
            ("dwg", dwg, dg.t() @ x.double(), dg.abs().t() @ x.double().abs(), T),
            ("dwu", dwu, du.t() @ x.double(), du.abs().t() @ x.double().abs(), T)):
        tiny = TINY[dtype] * (2 * F if name == "dx" else T) * 4  # gradients below the type's normal numbers
        close(got, want, rounded(want, dtype) + (1.01 * U[dtype] + (n + 8) * U32) * size + tiny, name)
        # in the 2-norm the roundings of operands and of the result are far from their bounds
        mag[name] = float((got.double() - want).norm() / want.norm())
        assert mag[name] <= 1.5 * U[dtype], (name, mag)
    again = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dwg, dwu)))


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_ff_by_differences(act):
    """<gradient, step> against the change of sum(dh * h) between two ends that the type holds exactly: curvature and the
    rounding of h to 11 bits stay within 3 % of a change along the gradient."""
    T, D, F = 50, 120, 90
    x, wg, wu, dh = gated_inputs(T, D, F, F16)
    saved = B.gated_ff_saved(T, F, DEV)
    B.bnn_gated_ff(x, wg, wu, act, saved=saved)
    grads = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    for i, size in ((0, 1.0), (1, 0.5), (2, 0.5)):
        if act == "relu" and i < 2:
            continue  # steps across its kink; h is linear in wu
        at = (x, wg, wu)[i]
        step = grads[i].double() / grads[i].double().norm()
        ends = [(at.double() + sign * size * step).half() for sign in (1, -1)]
        values = [float((dh.double() * B.bnn_gated_ff(*[end if k == i else (x, wg, wu)[k] for k in range(3)], act).double()).sum()) for end in ends]
        want = float(((ends[0].double() - ends[1].double()) * grads[i].double()).sum())
        assert abs(values[0] - values[1] - want) <= 0.03 * abs(want), (act, i, values, want)


@pytest.mark.parametrize("dtype,act,gap", [(BF16, "silu", 0), (F32, "gelu", 3), (F16, "gelu_tanh", 16)])
@pytest.mark.parametrize("T,D,F", GATED)
def test_gated_ff_i8(T, D, F, dtype, act, gap):
    print(f"gated i8 {T} x {D} x {F} {dtype} {act} gap {gap}", flush=True)
    g = gen(T, D, F, 8)
    x, wg, wu = (torch.randint(-128, 128, (n, D), generator=g, device=DEV, dtype=torch.int8) for n in (T, F, F))
    sx, sg, su = (torch.rand((n,), generator=g, device=DEV) * k + 0.1 * k for n, k in ((T, 0.02), (F, 1 / 74 / math.sqrt(D)), (F, 1 / 74 / math.sqrt(D))))
    rows = [strided(t, gap if gap % 16 else (-D) % 16 + gap) for t in (x, wg, wu)]
    room = torch.full((T, F + gap), 3.0, dtype=dtype, device=DEV)
    h = B.bnn_gated_ff_i8(rows[0], sx, rows[1], sg, rows[2], su, act, out=room[:, :F])
    zg = (x.double() @ wg.double().t()) * sx.double()[:, None] * sg.double()
    zu = (x.double() @ wu.double().t()) * sx.double()[:, None] * su.double()
    a, _ = act_ref(zg, act)
    want = a * zu
    off_a = 1.2 * 4 * U32 * zg.abs() + 16 * U32 * (zg.abs() + a.abs())
    close(h, want, rounded(want, dtype) + off_a * zu.abs() + 8 * U32 * want.abs(), "h")
    assert bool((room[:, F:] == 3.0).all())


def test_gated_ff_extreme_activations():
    """Projections far out on either side of the activations: no overflow of an intermediate shows in the result."""
    z = torch.tensor([[1e4], [-1e4], [300.0], [-300.0], [20.0], [-20.0], [0.0], [-0.0], [1e-30], [-1e-30]], device=DEV).to(BF16)
    one = torch.ones((1, 1), dtype=BF16, device=DEV)
    for act in ("silu", "gelu", "gelu_tanh", "relu"):
        saved = B.gated_ff_saved(10, 1, DEV)
        h = B.bnn_gated_ff(z, one, one, act, saved=saved)
        a, slope = act_ref(z.double(), act)
        close(h, a * z.double(), rounded(a * z.double(), BF16) + 32 * U32 * (z.double() ** 2 if act != "relu" else 0 * a) * (a != 0) + 1e-30, act)
        assert bool(saved.isfinite().all())


def test_empty_problems():
    e = torch.empty
    assert B.bnn_quant_rows_i8(e((0, 5), device=DEV))[0].shape == (0, 5)
    q, s = B.bnn_quant_rows_i8(normal(gen(1), 4, 32))
    assert B.bnn_linear_i8(q[:0], s[:0], q, s).shape == (0, 4) and B.bnn_linear_i8(q, s, q[:0], s[:0]).shape == (4, 0)
    x, wg, wu, dh = gated_inputs(4, 32, 24, BF16)
    assert B.bnn_gated_ff(x[:0], wg, wu).shape == (0, 24) and B.bnn_gated_ff(x, wg[:0], wu[:0]).shape == (4, 0)
    dx, dwg, dwu = B.bnn_gated_ff_backward(x[:0], wg, wu, B.gated_ff_saved(0, 24, DEV), dh[:0])
    assert dx.shape == (0, 32) and bool((dwg == 0).all()) and bool((dwu == 0).all())
    dx, dwg, dwu = B.bnn_gated_ff_backward(x, wg[:0], wu[:0], B.gated_ff_saved(4, 0, DEV), dh[:, :0])
    assert dwg.shape == (0, 32) and bool((dx == 0).all())


def test_other_streams():
    """Calls go to the current stream: a chain on another one, behind work that its inputs wait for."""
    stream = torch.cuda.Stream()
    x, wg, wu, _ = gated_inputs(300, 512, 520, BF16)
    want = B.bnn_gated_ff(x, wg, wu)
    wq = B.bnn_quant_rows_i8(normal(gen(2), 200, 520))
    want_y = B.bnn_linear_i8(*B.bnn_quant_rows_i8(want), *wq)
    torch.cuda.synchronize()
    late = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        busy = normal(gen(3), 4096, 4096)
        for _ in range(10):
            busy = busy @ busy * 1e-2
        late.copy_(x)
        h = B.bnn_gated_ff(late, wg, wu)
        y = B.bnn_linear_i8(*B.bnn_quant_rows_i8(h), *wq)
    stream.synchronize()
    assert torch.equal(h, want) and torch.equal(y, want_y)


def test_refusals_of_the_binding():
    x, wg, wu, dh = gated_inputs(6, 32, 24, BF16)
    q, s = B.bnn_quant_rows_i8(x)
    for error, call in (
            (TypeError, lambda: B.bnn_quant_rows_i8(x.double())), (TypeError, lambda: B.bnn_quant_rows_i8(x.cpu())),
            (ValueError, lambda: B.bnn_quant_rows_i8(x.t())), (ValueError, lambda: B.bnn_quant_rows_i8(x, scale=s[:3])),
            (ValueError, lambda: B.bnn_linear_i8(q, s, q[:, :16], s)), (ValueError, lambda: B.bnn_linear_i8(q, s[:2], q, s)),
            (TypeError, lambda: B.bnn_linear_i8(x, s, q, s)), (ValueError, lambda: B.bnn_linear_i8(q, s, q, s, out=x)),
            (ValueError, lambda: B.bnn_linear_i8(q, s, q, s, bias=s[:2])),
            (ValueError, lambda: B.bnn_gated_ff(x, wg, wu[:3])), (ValueError, lambda: B.bnn_gated_ff(x, wg, wu, act="tanh")),
            (TypeError, lambda: B.bnn_gated_ff(x, wg.half(), wu)), (ValueError, lambda: B.bnn_gated_ff(x, wg, wu, saved=s)),
            (B.BnnError, lambda: B.bnn_gated_ff(x.float(), wg.float(), wu.float())),
            (ValueError, lambda: B.bnn_gated_ff_backward(x, wg, wu, B.gated_ff_saved(6, 23, DEV), dh)),
            (B.BnnError, lambda: B.bnn_gated_ff_backward(x, wg, wu, B.gated_ff_saved(6, 24, DEV), dh,
                                                         workspace=torch.empty(64, dtype=torch.uint8, device=DEV))),
            (ValueError, lambda: B.bnn_norm_gate(x, x[:, :16])), (ValueError, lambda: B.bnn_norm_gate(x, x, post="batch")),
            (ValueError, lambda: B.bnn_norm_gate(x, x, w_pre=s)), (TypeError, lambda: B.bnn_norm_gate(x, x, gate=x.float())),
            (ValueError, lambda: B.bnn_norm_gate(x, x, gate=x, gate_rows=2)), (ValueError, lambda: B.bnn_norm_gate(x, x, gate=x, gate_rows=0)),
            (B.BnnError, lambda: B.bnn_norm_gate(x, x.half())), (B.BnnError, lambda: B.bnn_norm_gate(x, x, eps=-1.0)),
            (B.BnnError, lambda: B.bnn_norm_gate(x, x, pre="none", n_out=torch.empty_like(x))),
            (B.BnnError, lambda: B.bnn_norm_gate(x, x, q_out=q))):
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("post,pre,gate,vectors,dtype,rtype", NORM_KINDS)
def test_gradients_made_by_the_call_itself(post, pre, gate, vectors, dtype, rtype, monkeypatch):
    """The same tensors as where the binding makes room for them."""
    g = gen(post, pre)
    b, r, s = norm_inputs(g, 37, 200, dtype, rtype, post, pre, gate, vectors)
    dn = None if pre == "none" else strided(normal(g, 37, 200).to(dtype), 8)
    dr_out = strided(normal(g, 37, 200).to(rtype), 3)
    x, wg, wu, dh = gated_inputs(20, 72, 40, BF16)
    saved = B.gated_ff_saved(20, 40, DEV)
    B.bnn_gated_ff(strided(x, 8), wg, strided(wu, 16), saved=saved)
    norm = lambda: B.bnn_norm_gate_backward(b, r, dn, dr_out, **s)
    gated = lambda: dict(enumerate(B.bnn_gated_ff_backward(strided(x, 8), wg, strided(wu, 16), saved, dh)))
    got = norm(), gated()
    for name in ("norm_gate_gradients", "gated_ff_gradients"):
        monkeypatch.setattr(B._t(), name, lambda *args: None)
    for a, c in zip(got, (norm(), gated())):
        assert list(a) == list(c)
        for k in a:
            assert a[k].dtype == c[k].dtype and a[k].stride() == c[k].stride() and torch.equal(a[k], c[k]), k
