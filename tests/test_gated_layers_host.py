"""Argument checks of the 8-bit and gated layers: every refusal comes before a launch, so nothing here needs a GPU."""
import ctypes

import pytest

from paper_1911_04477_amd import binding as B

OK, NULL, SHAPE, STRIDE, ALIGN, WORKSPACE, HIP, UNSUPPORTED = range(8)
A, MIS = 4096, 4100  # addresses that are never read
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_quant_rows_refusals(L):
    f = L.bnn_quant_rows_i8
    assert f(A, BF16, -1, 8, 8, A, 16, A, None) == SHAPE
    assert f(A, BF16, 4, 0, 8, A, 16, A, None) == SHAPE
    assert f(A, 3, 4, 8, 8, A, 16, A, None) == SHAPE
    assert f(A, BF16, 4, 8, 7, A, 16, A, None) == STRIDE
    assert f(A, BF16, 4, 8, 8, A, 7, A, None) == STRIDE
    assert f(A, BF16, 4, 2 ** 31 - 1, 2 ** 31, A, 2 ** 31, A, None) == UNSUPPORTED
    assert f(None, BF16, 0, 8, 8, None, 8, None, None) == OK
    for bad in range(3):
        p = [A, A, A]
        p[bad] = None
        assert f(p[0], BF16, 4, 8, 8, p[1], 8, p[2], None) == NULL
        p[bad] = MIS
        assert f(p[0], BF16, 4, 8, 8, p[1], 8, p[2], None) == ALIGN


def test_linear_refusals(L):
    def f(M=4, N=5, K=6, lda=6, ldb=6, ldy=5, type=BF16, a=A, sa=A, b=A, sb=A, bias=None, y=A):
        return L.bnn_linear_i8(a, lda, sa, b, ldb, sb, bias, M, N, K, y, type, ldy, None)

    assert f(M=-1) == f(N=-1) == f(K=0) == f(type=3) == f(type=-1) == SHAPE
    assert f(lda=5) == f(ldb=5) == f(ldy=4) == STRIDE
    assert f(K=131072, lda=131072, ldb=131072) == f(M=2 ** 31 - 256) == f(N=2 ** 31 - 255, ldy=2 ** 31) == UNSUPPORTED
    assert f(M=0, a=None, sa=None, b=None, sb=None, y=None) == f(N=0, a=None, y=None) == OK
    for name in ("a", "sa", "b", "sb", "y"):
        assert f(**{name: None}) == NULL and f(**{name: MIS}) == ALIGN
    assert f(bias=MIS) == ALIGN


def norm_in(**kw):
    given = dict(rows=4, D=8, type=BF16, r_type=BF16, post=1, pre=1, eps=1e-6, b=A, b_ld=8, r=A, r_ld=8)
    given.update(kw)
    return B.NormGateIn(**given)


def test_norm_gate_refusals(L):
    def f(r_out=A, r_out_ld=8, n=A, n_ld=8, q=None, q_ld=0, qs=None, **kw):
        return L.bnn_norm_gate(ctypes.byref(norm_in(**kw)), r_out, r_out_ld, n, n_ld, q, q_ld, qs, None)

    assert L.bnn_norm_gate(None, A, 8, A, 8, None, 0, None, None) == NULL
    for kw in (dict(rows=-1), dict(D=0), dict(type=3), dict(r_type=-1), dict(post=3), dict(pre=-1), dict(eps=-1e-6), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(gate=A, gate_ld=8, gate_rows=0), dict(post=0, w_post=A), dict(pre=0, bias_pre=A, n=None),
               dict(pre=0)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(b_ld=7), dict(r_ld=7), dict(gate=A, gate_ld=7, gate_rows=1), dict(r_out_ld=7), dict(n_ld=7), dict(q=A, qs=A, q_ld=7)):
        assert f(**kw) == STRIDE, kw
    for kw in (dict(r_type=F16), dict(type=F32), dict(D=16385, b_ld=16385, r_ld=16385, r_out_ld=16385, n_ld=16385), dict(rows=2 ** 31)):
        assert f(**kw) == UNSUPPORTED, kw
    for kw in (dict(r=None), dict(r_out=None), dict(n=None), dict(q=A, q_ld=8), dict(qs=A), dict(b=None), dict(b=None, post=0),
               dict(b=None, post=0, r_out=None, res_scale=A)):
        assert f(**kw) == NULL, kw
    for kw in (dict(b=MIS), dict(r=MIS), dict(r_out=MIS), dict(n=MIS), dict(q=MIS, q_ld=8, qs=A), dict(q=A, q_ld=8, qs=MIS), dict(w_post=MIS),
               dict(w_pre=MIS), dict(bias_post=MIS), dict(bias_pre=MIS), dict(res_scale=MIS), dict(gate=MIS, gate_ld=8, gate_rows=2)):
        assert f(**kw) == ALIGN, kw
    assert f(rows=0, b=None, r=None, r_out=None, n=None) == OK
    assert f(b=None, post=0, pre=0, r_out=None, n=None) == OK  # nothing to write


def test_norm_gate_backward_refusals(L):
    def f(dn=A, dro=A, dr=A, db=A, dgate=None, sums=(None,) * 5, lds=(8,) * 5, ws=A, nbytes=None, **kw):
        p = norm_in(**kw)
        need = L.bnn_norm_gate_backward_workspace_bytes(p.rows, p.D, p.gate_rows if p.gate else 0)
        return L.bnn_norm_gate_backward(ctypes.byref(p), dn, lds[0], dro, lds[1], dr, lds[2], db, lds[3], dgate, lds[4], *sums, ws,
                                        need if nbytes is None else nbytes, None)

    assert f(rows=-1) == f(pre=0) == f(dgate=A) == f(pre=0, dn=None, sums=(None, None, None, A, None)) == SHAPE
    assert f(b=None, post=0) == SHAPE  # db of no b
    for i in range(4):
        assert f(lds=tuple(7 if k == i else 8 for k in range(5))) == STRIDE
    assert f(dr=None) == f(db=None) == f(r=None) == f(sums=(A, None, None, None, None), ws=None) == NULL
    assert f(sums=(None, A, None, None, None), nbytes=64) == WORKSPACE
    assert f(dgate=A, gate=A, gate_ld=8, gate_rows=4, nbytes=16) == WORKSPACE
    assert f(dn=MIS) == f(dro=MIS) == f(dr=MIS) == f(db=MIS) == f(ws=MIS) == f(sums=(None, None, MIS, None, None)) == ALIGN
    assert f(D=16385, b_ld=16385, r_ld=16385) == UNSUPPORTED
    assert f(rows=0, dr=None, db=None) == OK
    size = L.bnn_norm_gate_backward_workspace_bytes
    assert size(0, 8, 0) == size(4, 0, 0) == size(4, 16385, 0) == size(4, 8, -1) == 0
    assert size(1, 4096, 0) == 6 * 4 * 4096


def test_gated_refusals(L):
    def f(T=4, D=8, F=16, lds=(8, 8, 8, 16), type=BF16, act=0, x=A, wg=A, wu=A, h=A, saved=None):
        return L.bnn_gated_ff(x, lds[0], wg, lds[1], wu, lds[2], type, T, D, F, act, h, lds[3], saved, None)

    assert f(T=-1) == f(F=-1) == f(D=0) == f(act=4) == f(act=-1) == f(type=3) == SHAPE
    for i in range(4):
        assert f(lds=tuple(v - (k == i) for k, v in enumerate((8, 8, 8, 16)))) == STRIDE
    assert f(type=F32) == f(T=1 << 22) == f(F=1 << 22, lds=(8, 8, 8, 1 << 22)) == f(D=1 << 22, lds=(1 << 22,) * 4) == UNSUPPORTED
    assert f(T=0, x=None, h=None) == f(F=0, wg=None) == OK
    for name in ("x", "wg", "wu", "h"):
        assert f(**{name: None}) == NULL and f(**{name: MIS}) == ALIGN
    assert f(saved=MIS) == ALIGN
    assert L.bnn_gated_ff_saved_bytes(3, 5) == 120 and L.bnn_gated_ff_saved_bytes(0, 5) == L.bnn_gated_ff_saved_bytes(1 << 22, 5) == 0


def test_gated_i8_refusals(L):
    def f(T=4, D=8, F=16, lds=(8, 8, 8, 16), type=BF16, act=0, **kw):
        p = {**dict(x=A, sx=A, wg=A, sg=A, wu=A, su=A, h=A), **kw}
        return L.bnn_gated_ff_i8(p["x"], lds[0], p["sx"], p["wg"], lds[1], p["sg"], p["wu"], lds[2], p["su"], T, D, F, act, p["h"], type,
                                 lds[3], None)

    assert f(T=-1) == f(F=-1) == f(D=0) == f(act=4) == f(type=3) == SHAPE
    for i in range(4):
        assert f(lds=tuple(v - (k == i) for k, v in enumerate((8, 8, 8, 16)))) == STRIDE
    assert f(D=131072, lds=(131072,) * 4) == f(T=1 << 22) == UNSUPPORTED
    assert f(T=0, x=None) == OK
    for name in ("x", "sx", "wg", "sg", "wu", "su", "h"):
        assert f(**{name: None}) == NULL and f(**{name: MIS}) == ALIGN


def test_gated_backward_refusals(L):
    def f(T=4, D=8, F=16, lds=(8, 8, 8, 16, 8, 8, 8), type=BF16, nbytes=None, **kw):
        p = {**dict(x=A, wg=A, wu=A, saved=A, dh=A, dx=A, dwg=A, dwu=A, ws=A), **kw}
        need = L.bnn_gated_ff_backward_workspace_bytes(T, D, F)
        return L.bnn_gated_ff_backward(p["x"], lds[0], p["wg"], lds[1], p["wu"], lds[2], type, T, D, F, p["saved"], p["dh"], lds[3], p["dx"],
                                       lds[4], p["dwg"], lds[5], p["dwu"], lds[6], p["ws"], need if nbytes is None else nbytes, None)

    assert f(T=-1) == f(F=-1) == f(D=0) == f(type=3) == SHAPE
    for i in range(7):
        assert f(lds=tuple(v - (k == i) for k, v in enumerate((8, 8, 8, 16, 8, 8, 8)))) == STRIDE
    assert f(type=F32) == f(T=1 << 22) == UNSUPPORTED
    for name in ("x", "wg", "wu", "saved", "dh", "dx", "dwg", "dwu", "ws"):
        assert f(**{name: None}) == NULL and f(**{name: MIS}) == ALIGN, name
    assert f(nbytes=L.bnn_gated_ff_backward_workspace_bytes(4, 8, 16) - 1) == WORKSPACE
    assert f(T=0, F=0, dx=None, dwg=None, dwu=None) == OK
    assert L.bnn_gated_ff_backward_workspace_bytes(0, 8, 8) == L.bnn_gated_ff_backward_workspace_bytes(8, 8, 1 << 22) == 0


def test_calls_from_tensors_decline_what_is_not_plain():
    """CPU tensors, wrong counts and kinds of arguments are left to the binding, which raises."""
    import torch
    t = B._t()
    x, v, q = torch.zeros(4, 8), torch.zeros(4), torch.zeros(4, 8, dtype=torch.int8)
    none = [None] * 7
    for name, args in (("quant_rows", (x, q, v)), ("quant_rows", (x, q)), ("linear_i8", (q, v, q, v, None, x)),
                       ("norm_gate", (x, x, None, 1, *none[:5], 1, 1, 1e-6, x, x, None, None)), ("norm_gate", (x, x)),
                       ("norm_gate_backward", (x, x, None, 1, *none[:5], 1, 1, 1e-6, x, x, x, x, *none[:6], x)),
                       ("gated_ff", (x, x, x, 0, x, None)), ("gated_ff", (x, x, x, "silu", x, None)),
                       ("gated_ff_i8", (q, v, q, v, q, v, 0, x)), ("gated_ff_backward", (x, x, x, x, x, x, x, x, x))):
        assert getattr(t, name)(*args) is None, name
    with pytest.raises(TypeError):
        B.bnn_quant_rows_i8(x)
    with pytest.raises(TypeError):
        B.bnn_gated_ff(x, x, x)
