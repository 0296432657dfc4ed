"""Gradients of the norms around a block through the C ABI: every sum that a caller may ask for, whatever vectors it gave.

u is 2^-24; a sum of n fp32 terms is off by at most n u times the sum of their magnitudes."""
import ctypes
import zlib

import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U32 = 2.0 ** -24
EPS = 1e-6
SUMS = ("dres_scale", "dw_post", "dbias_post", "dw_pre", "dbias_pre")
KINDS = {"none": 0, "rms": 1, "layer": 2}


def gen(*key):
    g = torch.Generator(device=DEV)
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def backward(b, r, dn, dro, post, pre, vectors, want, workspace=None):
    """bnn_norm_gate_backward in fp32 with the sums of `want` -> (dr, db, {name: sum})."""
    rows, D = r.shape
    vec = {k: v.data_ptr() for k, v in vectors.items()}
    p = B.NormGateIn(rows=rows, D=D, type=0, r_type=0, post=KINDS[post], pre=KINDS[pre], eps=EPS, b=b.data_ptr(), b_ld=D, r=r.data_ptr(),
                     r_ld=D, **vec)
    dr, db = torch.empty_like(r), torch.empty_like(b)
    sums = {k: torch.full((D,), float("nan"), device=DEV) for k in want}
    ws = torch.empty(max(16, B.norm_gate_backward_workspace_bytes(rows, D, 0)), dtype=torch.uint8, device=DEV)
    st = B.lib().bnn_norm_gate_backward(ctypes.byref(p), dn.data_ptr(), D, dro.data_ptr(), D, dr.data_ptr(), D, db.data_ptr(), D, None, 0,
                                        *[sums[k].data_ptr() if k in sums else None for k in SUMS], ws.data_ptr(), ws.numel(),
                                        torch.cuda.current_stream().cuda_stream)
    assert st == 0, st
    return dr, db, sums


def unit(x, norm):
    if norm == "none":
        return x, torch.ones_like(x[:, :1])
    if norm == "layer":
        x = x - x.mean(1, keepdim=True)
    rs = 1 / (x.square().mean(1, keepdim=True) + EPS).sqrt()
    return x * rs, rs


def reference(b, r, dn, dro, post, pre, vectors):
    """In 64 bits: the sums, and what each may be off by.  A row's chain of about twenty operations and sums of at most 40 partial
    sums a value is off by at most 256 u of its terms' magnitudes, the sum over the rows by its length."""
    one = torch.ones((b.shape[1],), dtype=torch.float64, device=DEV)
    v = {k: vectors[k].double() if k in vectors else one * (0.0 if k.startswith("bias") else 1.0)
         for k in ("res_scale", "w_post", "bias_post", "w_pre", "bias_pre")}
    b, r, dn, dro = (t.double() for t in (b, r, dn, dro))
    ub, rsb = unit(b, post)
    p = ub * v["w_post"] + v["bias_post"]
    r1 = r + v["res_scale"] * p
    ur, rsr = unit(r1, pre)
    e = dn * v["w_pre"]
    level = e.mean(1, keepdim=True) if pre == "layer" else 0.0
    dr = dro + (e if pre == "none" else rsr * (e - level - ur * (e * ur).mean(1, keepdim=True)))
    dp = dr * v["res_scale"]
    terms = {"dres_scale": dr * p, "dw_post": dp * ub, "dbias_post": dp, "dw_pre": dn * ur, "dbias_pre": dn}
    # magnitudes of what dr, ub and ur are made of: means of magnitudes stand for centred values
    mean = lambda t: t.abs().mean(1, keepdim=True)
    size_ub, size_ur = ub.abs() + rsb * mean(b), ur.abs() + rsr * (mean(r1) + r.abs() + (v["res_scale"] * p).abs())
    size_dr = dro.abs() + rsr * (e.abs() + mean(e) + size_ur * (e.abs() * size_ur).mean(1, keepdim=True))
    size_dp = size_dr * v["res_scale"].abs()
    sizes = {"dres_scale": size_dr * (size_ub * v["w_post"].abs() + v["bias_post"].abs()), "dw_post": size_dp * size_ub,
             "dbias_post": size_dp, "dw_pre": dn.abs() * size_ur, "dbias_pre": dn.abs()}
    return {k: (t.sum(0), (256 + b.shape[0]) * U32 * sizes[k].sum(0)) for k, t in terms.items()}


@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "rms"), ("rms", "layer")])
@pytest.mark.parametrize("rows,D", [(37, 64), (5, 520), (700, 4096), (37, 2321), (40, 8192), (9, 16384)])
def test_sums_of_absent_vectors(rows, D, post, pre):
    """The gradient of a vector that is absent is the formula's at 1, or for a bias at 0."""
    print(f"absent vectors {rows} x {D} {post} {pre}", flush=True)
    g = gen(rows, D, post, pre)
    b, r, dn, dro = (torch.randn((rows, D), generator=g, device=DEV) for _ in range(4))
    want = reference(b, r, dn, dro, post, pre, {})
    dr, db, got = backward(b, r, dn, dro, post, pre, {}, SUMS)
    for k in SUMS:
        off = (got[k].double() - want[k][0]).abs()
        assert bool((off <= want[k][1]).all()), (k, float((off / want[k][1]).max()))
    for k in SUMS:  # one alone, and the rows' gradients with no sum at all
        alone = backward(b, r, dn, dro, post, pre, {}, (k,))
        off = (alone[2][k].double() - want[k][0]).abs()
        assert bool((off <= want[k][1]).all()), k
    bare = backward(b, r, dn, dro, post, pre, {}, ())
    for x, y in zip(bare[:2], (dr, db)):
        assert float((x - y).abs().max()) <= 1e-5 * float(y.abs().max())


@pytest.mark.parametrize("gate_rows", [1, 3, 700])
@pytest.mark.parametrize("rows,D", [(1, 4096), (40, 4097), (303, 2832), (700, 520), (140, 456)])
def test_gradient_of_the_gate_where_the_block_is_near_zero(rows, D, gate_rows):
    """p, the normed block's output, is off by u of what it is made of (the row's mean, the weight, the bias), not of itself, where they
    cancel; so is its product with the gradient of r'."""
    print(f"dgate {rows} x {D}, {gate_rows} rows a gate", flush=True)
    g = gen(rows, D, gate_rows)
    b, r, dn, dro = (torch.randn((rows, D), generator=g, device=DEV) + (0.5 if i == 0 else 0.0) for i in range(4))
    groups = -(-rows // gate_rows)
    gate, scale, w, bias = (torch.randn(s, generator=g, device=DEV) for s in ((groups, D), (D,), (D,), (D,)))
    got = B.bnn_norm_gate_backward(b, r, dn, dro, gate=gate, gate_rows=gate_rows, res_scale=scale, w_post=w, bias_post=bias, post="layer",
                                   pre="rms")["dgate"]
    at = torch.arange(rows, device=DEV) // gate_rows
    m = scale.double() * gate.double()[at]
    ub, rsb = unit(b.double(), "layer")
    p = ub * w.double() + bias.double()
    r1 = r.double() + m * p
    ur, rsr = unit(r1, "rms")
    e = dn.double()
    dr = dro.double() + rsr * (e - ur * (e * ur).mean(1, keepdim=True))
    size_p = (ub.abs() + rsb * b.double().abs().mean(1, keepdim=True)) * w.double().abs() + bias.double().abs()
    size_ur = ur.abs() + rsr * (r.double().abs() + m.abs() * size_p)
    size_dr = dro.double().abs() + rsr * (e.abs() + size_ur * (e.abs() * size_ur).mean(1, keepdim=True))
    zero = torch.zeros((groups, D), dtype=torch.float64, device=DEV)
    want = zero.index_add(0, at, dr * scale.double() * p)
    bound = (256 + rows) * U32 * zero.index_add(0, at, size_dr * scale.double().abs() * size_p)
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
