"""The gated feed-forward's gradients where those of its projections are larger or smaller than fp16 holds, against the
formulas in 64 bits.  u is 2^-11 for fp16, 2^-24 for fp32."""
import zlib

import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U16, U32, TINY = 2.0 ** -11, 2.0 ** -24, 2.0 ** -24


def gen(*key):
    g = torch.Generator(device=DEV)
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def inputs(T, D, F, dh_size, saved_size, w_size, x_size):
    g = gen(T, D, F, dh_size)
    n = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    return ((x_size * n(T, D)).half(), (w_size * n(F, D)).half(), (w_size * n(F, D)).half(), saved_size * n(2, T, F),
            (dh_size * n(T, F)).half())


def check(x, wg, wu, saved, dh, got, rows=slice(None)):
    """rows: the tokens that are compared, where others hold what no result can be compared with."""
    dg, du = dh.double() * saved[0].double(), dh.double() * saved[1].double()
    top = float(torch.stack([dg, du]).nan_to_num(0, 0, 0).abs().max())
    # rounded once (u each, or where the scale leaves them below the normal numbers 2^-24 of the largest), then summed in fp32
    parts = [("dx", got[0], dg @ wg.double() + du @ wu.double(), dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs(),
              (wg.double().abs() + wu.double().abs()).sum(0), 2 * dh.shape[1])]
    if rows == slice(None):
        for name, t, d in (("dwg", got[1], dg), ("dwu", got[2], du)):
            parts.append((name, t, d.t() @ x.double(), d.abs().t() @ x.double().abs(), x.double().abs().sum(0), dh.shape[0]))
    for name, t, want, size, spread, n in parts:
        bound = U16 * want.abs() + TINY + (1.01 * U16 + (n + 8) * U32) * size + top * 2.0 ** -24 * spread
        off = (t.double() - want).abs()
        at = rows if name == "dx" else slice(None)
        assert bool(t[at].isfinite().all()), (name, "not finite")
        assert bool((off <= bound)[at].all()), (name, float((off / bound)[at].max()))
        if rows == slice(None) and dh.numel() > 1000 and float(want.abs().mean()) > 2.0 ** -14:  # far from the smallest numbers
            assert float((t.double() - want).norm() / want.norm()) <= 1.5 * U16, name


SIZES = [(1, 8, 1), (20, 72, 40), (3, 1032, 4099), (300, 264, 520), (8200, 64, 72), (1000, 1024, 2321)]


@pytest.mark.parametrize("dh_size,saved_size,w_size,x_size", [(1e3, 300.0, 2e-4, 2e-4), (1e4, 1e4, 1e-6, 1e-6), (1.0, 1.0, 0.05, 1.0),
                                                              (1e-2, 1e-1, 1.0, 1.0), (2e-6, 1e-2, 3e3, 3e3), (1e-3, 1e-12, 6e4, 6e4)])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_gradients_beyond_the_type(T, D, F, dh_size, saved_size, w_size, x_size):
    print(f"gated range {T} x {D} x {F} dh {dh_size} saved {saved_size}", flush=True)
    x, wg, wu, saved, dh = inputs(T, D, F, dh_size, saved_size, w_size, x_size)
    wg, wu, x = (t.clamp(-6e4, 6e4) for t in (wg, wu, x))
    got = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    check(x, wg, wu, saved, dh, got)
    assert all(torch.equal(p, q) for p, q in zip(got, B.bnn_gated_ff_backward(x, wg, wu, saved, dh)))


def test_one_large_token():
    """A single product past 65504 among ordinary ones, at the ends of the problem."""
    for at in ((0, 0), (299, 519)):
        x, wg, wu, saved, dh = inputs(300, 264, 520, 1.0, 1.0, 0.05, 1.0)
        wg[at[1]], wu[at[1]], x[at[0]] = 1e-3, 1e-3, 1e-3
        dh[at], saved[0][at], saved[1][at] = 4e4, 50.0, 0.0
        check(x, wg, wu, saved, dh, B.bnn_gated_ff_backward(x, wg, wu, saved, dh))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_token_that_is_not_finite(bad):
    """It stays in its own row of dx; the scale goes by the finite values."""
    x, wg, wu, saved, dh = inputs(40, 72, 136, 1e3, 300.0, 1e-3, 1e-3)
    dh[7, 3] = bad
    dx, dwg, dwu = got = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
    check(x, wg, wu, saved, dh, got, rows=torch.arange(40, device=DEV) != 7)
    assert not bool(dx[7].isfinite().any()) and not bool(dwg[3].isfinite().any())


def test_zero_gradients():
    x, wg, wu, saved, dh = inputs(20, 72, 40, 1.0, 1.0, 1.0, 1.0)
    assert all(bool((t == 0).all()) for t in B.bnn_gated_ff_backward(x, wg, wu, saved, 0 * dh))


def test_replayed_from_a_graph():
    """The scale is found anew at every replay."""
    x, wg, wu, saved, dh = inputs(300, 264, 520, 1e3, 300.0, 1e-3, 1e-3)
    out = [torch.empty_like(t) for t in (x, wg, wu)]
    ws = torch.empty(B.gated_ff_backward_workspace_bytes(300, 264, 520), dtype=torch.uint8, device=DEV)
    call = lambda: B.bnn_gated_ff_backward(x, wg, wu, saved, dh, *out, workspace=ws)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    first = dh.clone()
    for size in (1.0, 1e-6, 1e-3, 1.0):
        dh.copy_(first * size)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = B.bnn_gated_ff_backward(x, wg, wu, saved, dh)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), size
