"""The sublayer classes of paper_1911_04477_amd.block and the ways a call takes to the library, against the single calls."""
import math

import pytest
import torch

from paper_1911_04477_amd import binding as B
from paper_1911_04477_amd.block import GatedBlock8, GatedProjections

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16 = torch.bfloat16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def sublayer(T, D, F, seed=1):
    g = gen(seed)

    def n(*shape, std=1.0):
        return std * torch.randn(shape, generator=g, device=DEV)

    w = [n(F, D, std=D ** -0.5).to(BF16), n(F, D, std=D ** -0.5).to(BF16), n(D, F, std=F ** -0.5).to(BF16)]
    vectors = dict(res_scale=n(D), w_post=1 + 0.1 * n(D), w_pre=1 + 0.1 * n(D), post="rms", pre="rms", eps=1e-5)
    return w, vectors, n(T, D).to(BF16), n(T, D).to(BF16), n(1, D).to(BF16)


def norm64(x, eps):
    return x / (x.square().mean(1, keepdim=True) + eps).sqrt()


@pytest.mark.parametrize("T", [1, 7, 64, 130])
def test_serving_sublayer(T):
    """Against the sublayer in 64 bits without any quantization: rounding to 8 bits costs a product of K terms a relative
    error of about 1 / (127 sqrt 3) * (largest / rms) a factor, 1.5 % here; two products in a row stay below 6 %."""
    D, F = 328, 520
    w, v, b, r, gate = sublayer(T, D, F)
    net = GatedBlock8(*w, tokens=130, vectors=v)
    o, r1 = net.forward(b, r, gate, T)
    x = [t.double() for t in w]
    want_r = r.double() + v["res_scale"].double() * gate.double() * (norm64(b.double(), 1e-5) * v["w_post"].double())
    n = norm64(want_r, 1e-5) * v["w_pre"].double()
    want = (torch.nn.functional.silu(n @ x[0].t()) * (n @ x[1].t())) @ x[2].t()
    assert float((r1.double() - want_r).norm() / want_r.norm()) < 2.0 ** -8
    assert float((o.double() - want).norm() / want.norm()) < 0.06
    # tokens do not see each other: the same token alone gives the same bits
    alone = net.forward(b[T - 1:], r[T - 1:], gate, 1)[0].clone()  # the next pass writes the buffer again
    assert torch.equal(alone[0], net.forward(b, r, gate, T)[0][T - 1])
    first, stream = net.forward(None, r)
    n = norm64(r.double(), 1e-5) * v["w_pre"].double()
    want = (torch.nn.functional.silu(n @ x[0].t()) * (n @ x[1].t())) @ x[2].t()
    assert stream is r and float((first.double() - want).norm() / want.norm()) < 0.06
    with pytest.raises(ValueError):
        net.forward(torch.cat([b] * 131)[:131], torch.cat([r] * 131)[:131])


def test_serving_sublayer_in_a_graph():
    """Captured once, replayed on new inputs, with eager work between the replays."""
    T, D, F = 5, 256, 384
    w, v, b, r, gate = sublayer(T, D, F)
    net, r_out = GatedBlock8(*w, tokens=T, vectors=v), torch.empty_like(r)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        net.forward(b, r, gate, T, r_out)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        o, _ = net.forward(b, r, gate, T, r_out)
    other = GatedBlock8(*w, tokens=T, vectors=v)
    for k in range(4):
        _, _, b2, r2, _ = sublayer(T, D, F, seed=10 + k)
        b.copy_(b2), r.copy_(r2)
        graph.replay()
        torch.cuda.synchronize()
        got, got_r = o.clone(), r_out.clone()
        want, want_r = other.forward(b2, r2, gate, T)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(got_r, want_r), k


def test_training_pass():
    """Gradients of norms and projections together against torch's derivatives of the same formulas in 64 bits: every rounding
    to bf16 on the way (n, the projections' gradients, dn, the results) is 2^-8 at most, in the 2-norm 2 % in all."""
    T, D, F = 150, 200, 330
    (wg, wu, _), v, b, r, _ = sublayer(T, D, F)
    g = gen(5)
    gate = torch.rand((3, D), generator=g, device=DEV).to(BF16)
    dh, dro = (torch.randn(s, generator=g, device=DEV).to(BF16) for s in ((T, F), (T, D)))
    net = GatedProjections(wg, wu, v, act="gelu")
    h, r1 = net.forward(b, r, gate, 50)
    got = net.backward(dh, dro)
    leaves = {k: t.double().requires_grad_() for k, t in dict(b=b, r=r, gate=gate, wg=wg, wu=wu, res_scale=v["res_scale"],
                                                              w_post=v["w_post"], w_pre=v["w_pre"]).items()}
    L = leaves
    want_r = L["r"] + L["res_scale"] * L["gate"].repeat_interleave(50, 0) * (norm64(L["b"], 1e-5) * L["w_post"])
    n = norm64(want_r, 1e-5) * L["w_pre"]
    z = n @ L["wg"].t()
    want_h = 0.5 * z * (1 + torch.erf(z / math.sqrt(2))) * (n @ L["wu"].t())
    ((want_h * dh.double()).sum() + (want_r * dro.double()).sum()).backward()
    assert set(got) == {"d" + k for k in leaves}
    for k, t in leaves.items():
        off = float((got["d" + k].double() - t.grad).norm() / t.grad.norm())
        assert off < 0.02, (k, off)
    assert float((h.double() - want_h.detach()).norm() / want_h.detach().norm()) < 0.02
    with pytest.raises(RuntimeError):
        net.backward(dh, dro)


def test_both_ways_to_the_library(monkeypatch):
    """Calls from tensors and through ctypes' arguments give the same results."""
    D, F, T = 200, 136, 40
    w, v, b, r, gate = sublayer(T, D, F)
    dh, dro, dn = (torch.randn(s, device=DEV).to(BF16) for s in ((T, F), (T, D), (T, D)))

    def everything():
        q, qs = B.bnn_quant_rows_i8(b, B.rows_i8(T, D, DEV), torch.empty((T,), device=DEV))
        wq = B.bnn_quant_rows_i8(w[0])
        y = B.bnn_linear_i8(q, qs, *wq, bias=torch.ones((F,), device=DEV), out=torch.empty((T, F), device=DEV))
        h8 = B.bnn_gated_ff_i8(q, qs, *wq, *B.bnn_quant_rows_i8(w[1]), act="relu", out=torch.empty((T, F), dtype=BF16, device=DEV))
        saved = B.gated_ff_saved(T, F, DEV)
        h = B.bnn_gated_ff(b, w[0], w[1], out=torch.empty((T, F), dtype=BF16, device=DEV), saved=saved)
        grads = B.bnn_gated_ff_backward(b, w[0], w[1], saved, dh)
        r1, n = B.bnn_norm_gate(b, r, gate=gate, gate_rows=T, **v)
        back = B.bnn_norm_gate_backward(b, r, dn, dro, gate=gate, gate_rows=T, **v)
        return [q, qs, y, h8, h, saved, *grads, r1, n, *[back[k] for k in sorted(back)]]

    fast = everything()
    class Declines:
        def __getattr__(self, name):
            return lambda *args: None

    monkeypatch.setattr(B, "_t", Declines)
    for a, c in zip(fast, everything()):
        assert torch.equal(a, c)


def test_kernels_by_size():
    """Each form of the products is reached by a size of its own, and launches what it says."""
    B.prof_enable(True)
    try:
        for M, N, K, names in ((16, 64, 64, ["linear_i8_few"]), (17, 64, 64, ["linear_i8"])):
            a, b = (B.bnn_quant_rows_i8(torch.randn(n, K, device=DEV)) for n in (M, N))
            B.prof_reset()
            B.bnn_linear_i8(*a, *b)
            assert [n for n, _ in B.prof_records()] == names
        x, w, dh = (torch.randn(s, device=DEV).to(BF16) for s in ((70, 64), (128, 64), (70, 128)))
        saved = B.gated_ff_saved(70, 128, DEV)
        B.prof_reset()
        B.bnn_gated_ff(x, w, w, saved=saved)
        B.bnn_gated_ff_backward(x, w, w, saved, dh)
        assert [n for n, _ in B.prof_records()] == ["gated_ff", "gated_gradient", "gated_ff_backward", "gated_ff_backward"]
        odd = torch.randn(70, 63, device=DEV).to(BF16)
        ow = torch.randn(128, 63, device=DEV).to(BF16)
        B.prof_reset()
        B.bnn_gated_ff_backward(odd, ow, ow, saved, dh)
        assert [n for n, _ in B.prof_records()].count("realign") == 3
        long = [torch.randn(s, device=DEV).to(BF16) for s in ((8, 64), (8192, 64), (8192, 64), (8, 8192))]
        saved = B.gated_ff_saved(8, 8192, DEV)
        B.bnn_gated_ff(*long[:3], saved=saved)
        B.prof_reset()
        B.bnn_gated_ff_backward(*long[:3], saved, long[3])
        assert "product_sums" in [n for n, _ in B.prof_records()]  # few tiles: k in shares
    finally:
        B.prof_enable(False)


@pytest.mark.parametrize("T,D,F", [(1, 64, 8200), (3, 1032, 4099), (100, 72, 20000), (8200, 64, 64), (8200, 65, 66), (700, 200, 3001)])
def test_gated_backward_in_shares(T, D, F):
    """Long reductions that are split over workgroups, with what is left of k in the last share: 2-norm bound of the operands'
    and the results' roundings (2^-8 each at most, far less on average), and the same bits twice."""
    g = gen(T + F)
    x, wg, wu, dh = (torch.randn(s, generator=g, device=DEV).to(BF16) for s in ((T, D), (F, D), (F, D), (T, F)))
    saved = torch.randn((2, T, F), generator=g, device=DEV)
    got = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    dg, du = (dh.double() * s.double() for s in saved)
    for a, want in zip(got, (dg @ wg.double() + du @ wu.double(), dg.t() @ x.double(), du.t() @ x.double())):
        assert float((a.double() - want).norm() / want.norm()) < 1.5 * 2.0 ** -8
    assert all(torch.equal(a, c) for a, c in zip(got, B.bnn_gated_ff_backward(x, wg, wu, saved, dh)))


@pytest.mark.parametrize("M,N,K", [(4096, 8192, 128), (4096, 8192, 200), (8192, 4104, 384), (1024, 3001, 2321), (520, 4096, 1000),
                                   (256, 4096, 4096), (100, 4096, 513), (64, 8192, 4100), (33, 4096, 130)])
def test_products_of_every_form(M, N, K):
    """Sums are exact in 8 bits: every tile form, over many and few steps, whole and cut short, equals the product in 64 bits."""
    g = gen(M + N + K)
    a, b = (torch.randint(-128, 128, (n, K), generator=g, device=DEV, dtype=torch.int8) for n in (M, N))
    one = torch.ones((max(M, N),), device=DEV)
    padded = [B.rows_i8(n, K, DEV) for n in (M, N)]
    padded[0].copy_(a), padded[1].copy_(b)
    want = (a.double() @ b.double().t()).float()
    assert torch.equal(B.bnn_linear_i8(padded[0], one[:M], padded[1], one[:N], dtype=torch.float32), want)
    if K % 16:
        assert torch.equal(B.bnn_linear_i8(a, one[:M], b, one[:N], dtype=torch.float32), want)  # rows at any address
