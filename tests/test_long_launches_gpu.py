"""Sizes beyond 32 bits: workgroups of 2^32 threads and more, which one dimension of a launch does not take (rows of the quantizer, columns of
the 8-bit product with few rows and with tiles), matrices past 2^32 bytes, and tiles whose rows lie further apart than 2^31."""
import gated_forms
import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def check_rows(rows, K, dtype):
    """The same few rows again and again, the last ones cut off."""
    g = torch.Generator(device=DEV)
    g.manual_seed(K)
    some = torch.randn((1 << 16, K), generator=g, device=DEV).to(dtype)
    want, want_s = (t.clone() for t in B.bnn_quant_rows_i8(some))
    whole = -(-rows // some.shape[0])
    x = some.expand(whole, *some.shape).reshape(-1, K)[:rows]
    q, s = torch.full((rows, K), 99, dtype=torch.int8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    B.bnn_quant_rows_i8(x, q, s)
    for i in range(whole):
        a, b = i << 16, min(rows, (i + 1) << 16)
        if i % 16 == 0 or i + 2 >= whole:
            assert torch.equal(q[a:b], want[:b - a]) and torch.equal(s[a:b], want_s[:b - a]), i
    assert bool((s >= 0).all())  # every row has been written


@pytest.mark.parametrize("rows,K,dtype", [((1 << 26) + 5, 3, torch.float16), ((1 << 26) + 70001, 8, torch.float32),
                                          ((1 << 25) + 12345, 520, torch.bfloat16)])
def test_rows_of_the_quantizer(rows, K, dtype):
    print(f"quant {rows} x {K}", flush=True)
    check_rows(rows, K, dtype)


@pytest.mark.parametrize("M,N", [(2, (1 << 27) + 37), (17, (1 << 29) + 100)])
def test_columns_of_the_8_bit_product(M, N):
    """One term a sum, exact in 16 bits: products of numbers up to 8."""
    print(f"linear {M} x {N}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(M)
    a = torch.randint(-8, 9, (M, 1), generator=g, device=DEV, dtype=torch.int8)
    b = torch.randint(-8, 9, (N, 1), generator=g, device=DEV, dtype=torch.int8)
    one = torch.ones((N,), device=DEV)
    y = torch.full((M, N), 99.0, dtype=torch.bfloat16, device=DEV)
    B.bnn_linear_i8(a, one[:M], b, one, out=y)
    bt = b.view(1, N).to(torch.bfloat16)
    for m in range(M):
        assert torch.equal(y[m:m + 1], bt * a[m].to(torch.bfloat16)), m


def pieces(n, step):
    return [(a, min(a + step, n)) for a in range(0, n, step)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gated_rows_past_32_bits(dtype):
    """h, what the forward pass saves and the projections' gradients each end past 2^32 bytes; rows at both ends of every tensor, and the
    weights' gradients, which add up all rows, against the formulas in 64 bits.  Bounds: test_gated_layers_gpu.py's, in the 2-norm."""
    T, D, F = 1100003, 72, 2056
    print(f"gated {T} x {D} x {F} {dtype}", flush=True)
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    x, wg, wu = n(T, D).to(dtype), (n(F, D) / D ** 0.5).to(dtype), (n(F, D) / D ** 0.5).to(dtype)
    dh = (n(1 << 16, F).to(dtype)).repeat(-(-T >> 16), 1)[:T]
    saved = B.gated_ff_saved(T, F, DEV)
    h = B.bnn_gated_ff(x, wg, wu, "silu", saved=saved)
    dx, dwg, dwu = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    want_g, want_u = (torch.zeros((F, D), dtype=torch.float64, device=DEV) for _ in range(2))
    off = lambda got, want: float((got.double() - want).norm() / want.norm())
    for a, b in pieces(T, 1 << 15):
        xs = x[a:b].double()
        zg, zu = xs @ wg.double().t(), xs @ wu.double().t()
        s = torch.sigmoid(zg)
        act, slope = zg * s, s * (1 + zg * (1 - s))
        d = dh[a:b].double()
        dg, du = d * zu * slope, d * act
        want_g += dg.t() @ xs
        want_u += du.t() @ xs
        if a % (1 << 18) == 0 or b + (1 << 16) > T:
            assert off(h[a:b], act * zu) < u and off(saved[0, a:b], zu * slope) < 1e-5 and off(saved[1, a:b], act) < 1e-5, a
            assert off(dx[a:b], dg @ wg.double() + du @ wu.double()) < 1.5 * u, a
    assert off(dwg, want_g) < 1.5 * u and off(dwu, want_u) < 1.5 * u


def test_norm_rows_past_32_bits():
    """Every matrix ends past 2^32 bytes; rows at both ends, and sums over all rows against the formula in 64 bits."""
    rows, D = 600001, 4096
    print(f"norm {rows} x {D}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    some = [torch.randn((1 << 14, D), generator=g, device=DEV).bfloat16() for _ in range(4)]
    b, r, dn, dro = (t.repeat(-(-rows >> 14), 1)[:rows] for t in some)
    w = 1 + 0.1 * torch.randn((D,), generator=g, device=DEV)
    r1, y = B.bnn_norm_gate(b, r, w_post=w, w_pre=w)
    back = B.bnn_norm_gate_backward(b, r, dn, dro, w_post=w, w_pre=w)
    few = slice(0, 1 << 14)
    want = (*B.bnn_norm_gate(b[few], r[few], w_post=w, w_pre=w), B.bnn_norm_gate_backward(b[few], r[few], dn[few], dro[few], w_post=w, w_pre=w))
    for a, c in pieces(rows, 1 << 14):  # the same rows again and again
        n = c - a
        assert torch.equal(r1[a:c], want[0][:n]) and torch.equal(y[a:c], want[1][:n]), a
        assert torch.equal(back["dr"][a:c], want[2]["dr"][:n]) and torch.equal(back["db"][a:c], want[2]["db"][:n]), a
    unit = lambda t: t / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()
    total, size = torch.zeros((D,), dtype=torch.float64, device=DEV), torch.zeros((D,), dtype=torch.float64, device=DEV)
    for a, c in pieces(rows, 1 << 12):
        e = dn[a:c].double() * unit(r[a:c].double() + unit(b[a:c].double()) * w.double())
        total, size = total + e.sum(0), size + e.abs().sum(0)
    # a team adds up to 2400 rows one after the other, the sums of 256 teams meet in 16 and in 16 steps; the terms are good to 256 u
    assert bool(((back["dw_pre"].double() - total).abs() <= (2400 + 32 + 256) * 2.0 ** -24 * size).all())


def test_gradients_in_rows_past_2_to_the_31():
    """A tile of 256 rows of gradients spans more than 2^31 bytes, and k ends in a remainder: dx, and the weights' gradients at both ends,
    against the formulas in 64 bits."""
    T, D, F = 300, 1024, 2200001
    print(f"gated backward {T} x {D} x {F}: {gated_forms.backward_plan(T, D, F)}", flush=True)
    (form, _), _, largest = gated_forms.backward_plan(T, D, F)
    assert form == 0 and largest > 2 ** 31
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    x, dh = n(T, D).bfloat16(), n(T, F).bfloat16()
    wg, wu = (torch.empty((F, D), dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    saved = torch.empty((2, T, F), device=DEV).normal_(generator=g)
    dx, dwg, dwu = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    off = lambda got, want: float((got.double() - want).norm() / want.norm())
    want = torch.zeros((T, D), dtype=torch.float64, device=DEV)
    xt = x.double()
    for a, b in pieces(F, 1 << 16):
        dg, du = (dh[:, a:b].double() * saved[i, :, a:b].double() for i in range(2))
        want += dg @ wg[a:b].double() + du @ wu[a:b].double()
        if a == 0 or b + (1 << 16) > F:
            assert off(dwg[a:b], dg.t() @ xt) < 1.5 * 2.0 ** -8 and off(dwu[a:b], du.t() @ xt) < 1.5 * 2.0 ** -8, a
    assert off(dx, want) < 1.5 * 2.0 ** -8
