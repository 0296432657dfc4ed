"""Argument checks of 8-bit floating point and experts: every refusal comes before a launch, so nothing here needs a GPU."""
import ctypes

import pytest
import torch

from paper_1911_04477_amd import binding as B

OK, NULL, SHAPE, STRIDE, ALIGN, WORKSPACE, HIP, UNSUPPORTED = range(8)
A, MIS, ODD = 4096, 4100, 4098  # addresses that are never read
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_sizes(L):
    assert [L.bnn_f8_row_bytes(k) for k in (-1, 0, 1, 128, 129)] == [0, 0, 128, 128, 256]
    assert [L.bnn_f8_scale_bytes(k) for k in (-1, 0, 1, 512, 513)] == [0, 0, 4, 4, 8]
    assert L.bnn_expert_rows(10, 2, 4, 1) == 20 and L.bnn_expert_rows(10, 2, 4, 128) == (20 + 4 * 127) // 128 * 128
    assert L.bnn_expert_rows(1, 2, 64, 8) == 16 and L.bnn_expert_rows(0, 2, 4, 8) == 0
    assert L.bnn_expert_sort_workspace_bytes(4, 2, 64) == 0 and L.bnn_expert_sort_workspace_bytes(2048, 2, 64) == 0
    assert L.bnn_expert_sort_workspace_bytes(2049, 2, 64) == 256 * 64 * 4


@pytest.mark.parametrize("name", ["bnn_quant_blocks_f8", "bnn_quant_columns_f8"])
def test_quant_refusals(L, name):
    columns = name == "bnn_quant_columns_f8"

    def f(x=A, type=BF16, T=4, x_ld=8, rows=None, k=1, S=4, K=8, q=A, q_ld=128, s=A, s_ld=4):
        return getattr(L, name)(x, type, T, x_ld, rows, k, S, K, q, q_ld, s, s_ld, None)

    assert f(T=-1) == f(S=-1, rows=A) == f(K=0) == f(type=3) == f(S=5) == f(rows=A, k=0) == SHAPE
    assert f(x_ld=7) == f(q_ld=127) == f(q_ld=136) == f(s_ld=3) == f(s_ld=6) == STRIDE
    assert f(K=2 ** 28 + 1, x_ld=2 ** 30) == f(rows=A, T=2 ** 20, k=2 ** 20) == f(rows=A, S=2 ** 31) == UNSUPPORTED
    assert f(T=0, S=0, x=None, q=None, s=None) == OK
    for arg, bad in (("x", MIS), ("q", MIS), ("s", ODD)):
        assert f(**{arg: None}) == NULL and f(**{arg: bad}) == ALIGN
    assert f(rows=ODD) == ALIGN
    if columns:
        assert f(rows=A, S=2 ** 22, q_ld=2 ** 22) == UNSUPPORTED
        assert f(rows=A, T=0, S=4) == SHAPE


def weight(q=A, ld=128, expert_ld=640, scale=A, scale_ld=4, scale_expert_ld=4):
    return B.F8Weight(q, ld, expert_ld, scale, scale_ld, scale_expert_ld)


def test_quant_weight_refusals(L):
    def f(w=A, type=BF16, E=2, es=40, N=5, K=8, ld=8, out=weight(), turned=weight(expert_ld=1024)):
        return L.bnn_quant_weight_f8(w, type, E, es, N, K, ld, out, turned, None)

    assert f(E=-1) == f(N=0) == f(K=0) == f(type=4) == SHAPE
    assert f(ld=7) == f(es=-1) == f(out=weight(ld=120)) == f(out=weight(expert_ld=639)) == f(out=weight(expert_ld=650)) == STRIDE
    assert f(turned=weight(expert_ld=1023)) == f(out=weight(scale_ld=2)) == f(out=weight(scale_expert_ld=2)) == STRIDE
    assert f(E=65536) == f(N=2 ** 22 + 1) == f(K=2 ** 22 + 1, ld=2 ** 23) == UNSUPPORTED
    assert f(w=None) == f(out=None, turned=None) == f(out=weight(q=None)) == f(turned=weight(scale=None, expert_ld=1024)) == NULL
    assert f(w=MIS) == f(out=weight(q=MIS)) == f(out=weight(scale=ODD)) == ALIGN
    assert f(E=0) == OK


def test_linear_refusals(L):
    def f(a=A, lda=256, sa=A, sa_ld=4, b=A, ldb=256, sb=A, kind=0, sb_ld=4, per=1, bias=None, M=4, N=5, K=200, y=A, type=BF16, ldy=5):
        return L.bnn_linear_f8(a, lda, sa, sa_ld, b, ldb, sb, kind, sb_ld, per, bias, M, N, K, y, type, ldy, None)

    assert f(M=-1) == f(N=-1) == f(K=0) == f(type=3) == f(kind=2) == f(per=2) == f(kind=1, per=1) == SHAPE
    assert f(lda=255) == f(lda=264) == f(ldb=128) == f(sa_ld=3) == f(sa_ld=5) == f(sb_ld=2) == f(ldy=4) == f(kind=1, per=128, sb_ld=1) == STRIDE
    assert f(M=2 ** 31 - 256) == f(N=2 ** 31 - 256, ldy=2 ** 31) == f(K=2 ** 22 + 1) == f(lda=2 ** 22) == UNSUPPORTED
    for arg, bad in (("a", MIS), ("sa", ODD), ("b", MIS), ("sb", ODD), ("y", MIS)):
        assert f(**{arg: None}) == NULL and f(**{arg: bad}) == ALIGN
    assert f(bias=ODD) == ALIGN
    assert f(M=0, a=None, y=None) == f(N=0, b=None, y=None) == OK


def test_expert_linear_refusals(L):
    def f(a=A, lda=256, sa=A, sa_ld=4, off=A, E=3, b=A, ldb=256, es=1280, sb=A, kind=0, sb_ld=4, sb_es=20, per=1, S=4, N=5, K=200, y=A,
          type=BF16, ldy=5):
        return L.bnn_expert_linear_f8(a, lda, sa, sa_ld, off, E, b, ldb, es, sb, kind, sb_ld, sb_es, per, S, N, K, y, type, ldy, None)

    assert f(S=-1) == f(N=-1) == f(K=0) == f(E=-1) == f(type=-1) == f(kind=3) == f(per=64) == SHAPE
    assert f(es=1279) == f(es=1288) == f(sb_es=19) == f(sb_es=22) == f(lda=0) == f(ldy=4) == f(kind=1, per=128, sb_es=3) == STRIDE
    assert f(E=65536) == f(S=2 ** 31) == f(ldb=2 ** 22, es=5 * 2 ** 22) == UNSUPPORTED
    for arg, bad in (("a", MIS), ("sa", ODD), ("off", ODD), ("b", MIS), ("sb", ODD), ("y", MIS)):
        assert f(**{arg: None}) == NULL and f(**{arg: bad}) == ALIGN
    assert f(S=0, a=None) == f(E=0, b=None) == f(N=0, y=None) == OK

    def g(a=A, lda=256, sa=A, sa_ld=4, b=A, ldb=256, sb=A, sb_ld=4, off=A, E=3, N=5, K=6, S=200, dw=A, type=F32, ld=6, es=30):
        return L.bnn_expert_linear_f8_dw(a, lda, sa, sa_ld, b, ldb, sb, sb_ld, off, E, N, K, S, dw, type, ld, es, None)

    assert g(S=-1) == g(N=-1) == g(K=-1) == g(E=-1) == g(type=3) == SHAPE
    assert g(ld=5) == g(es=29) == g(lda=128) == g(sb_ld=1) == STRIDE
    assert g(S=2 ** 22) == g(E=65536) == UNSUPPORTED
    for arg, bad in (("a", MIS), ("sa", ODD), ("b", MIS), ("sb", ODD), ("off", ODD), ("dw", MIS)):
        assert g(**{arg: None}) == NULL and g(**{arg: bad}) == ALIGN
    assert g(E=0, dw=None) == g(N=0, dw=None) == g(K=0, dw=None) == OK


def test_sort_refusals(L):
    def f(e=A, size=4, T=10, k=2, E=4, align=1, S=20, off=A, rows=A, places=A, ws=None, nbytes=0):
        return L.bnn_expert_sort(e, size, T, k, E, align, S, off, rows, places, ws, nbytes, None)

    assert f(T=-1) == f(k=0) == f(E=0) == f(align=0) == f(S=-1) == f(size=2) == f(S=19) == f(align=128, S=383) == SHAPE
    assert f(E=1025) == f(align=4097) == f(T=2 ** 20, k=2 ** 11) == f(S=2 ** 31) == UNSUPPORTED
    assert f(e=None) == f(off=None) == f(rows=None) == f(places=None) == NULL
    assert f(e=ODD) == f(e=MIS, size=8) == f(off=ODD) == f(rows=ODD) == f(places=ODD) == ALIGN
    need = L.bnn_expert_sort_workspace_bytes(3000, 2, 4)
    assert f(T=3000, S=6000, ws=A, nbytes=need - 1) == WORKSPACE
    assert f(T=3000, S=6000, ws=None, nbytes=need) == NULL and f(T=3000, S=6000, ws=MIS, nbytes=need) == ALIGN


def test_sizes_of_refused_sorts(L):
    """Products of sizes past 64 bits, and experts that the sort does not take, ask for nothing."""
    for T, k, E in ((2 ** 40, 2 ** 40, 8), (2 ** 20, 2 ** 11, 8), (2 ** 62, 3, 1), (4096, 2, 1025), (-1, 2, 8)):
        assert L.bnn_expert_sort_workspace_bytes(T, k, E) == L.bnn_expert_rows(T, k, E, 1) == 0
    assert L.bnn_expert_sort_workspace_bytes(2 ** 20, 2 ** 10, 1024) > 0 and L.bnn_expert_rows(2 ** 20, 2 ** 10, 1024, 1) == 2 ** 30


def test_gather_and_combine_refusals(L):
    def g(x=A, type=BF16, T=4, ld=8, rows=A, k=2, S=8, D=8, xs=A, xs_ld=8):
        return L.bnn_expert_gather(x, type, T, ld, rows, k, S, D, xs, xs_ld, None)

    assert g(T=-1) == g(S=-1) == g(D=0) == g(k=0) == g(type=3) == SHAPE
    assert g(ld=7) == g(xs_ld=7) == STRIDE
    assert g(D=2 ** 28 + 1, ld=2 ** 29, xs_ld=2 ** 29) == g(T=2 ** 20, k=2 ** 11) == UNSUPPORTED
    assert g(x=None) == g(rows=None) == g(xs=None) == NULL and g(x=MIS) == g(rows=ODD) == g(xs=MIS) == ALIGN
    assert g(S=0, x=None, rows=None, xs=None) == OK

    def c(ys=A, type=BF16, S=8, ld=8, places=A, w=None, T=4, k=2, D=8, out=A, out_ld=8):
        return L.bnn_expert_combine(ys, type, S, ld, places, w, T, k, D, out, out_ld, None)

    assert c(T=-1) == c(S=-1) == c(D=0) == c(k=0) == c(type=3) == SHAPE
    assert c(ld=7) == c(out_ld=7) == STRIDE
    assert c(ys=None) == c(places=None) == c(out=None) == NULL and c(ys=MIS) == c(places=ODD) == c(w=ODD) == c(out=MIS) == ALIGN
    assert c(T=0, ys=None, places=None, out=None) == OK

    def b(ys=A, type=BF16, S=8, ld=8, rows=A, places=A, w=None, dout=A, dout_ld=8, T=4, k=2, D=8, dys=A, dys_ld=8, dw=A):
        return L.bnn_expert_combine_backward(ys, type, S, ld, rows, places, w, dout, dout_ld, T, k, D, dys, dys_ld, dw, None)

    assert b(T=-1) == b(S=-1) == b(D=0) == b(k=0) == b(type=3) == SHAPE
    assert b(ld=7) == b(dout_ld=7) == b(dys_ld=7) == STRIDE
    assert b(D=32769, ld=32769, dout_ld=32769, dys_ld=32769) == UNSUPPORTED
    assert b(ys=None) == b(rows=None) == b(places=None) == b(dout=None) == b(dys=None, dw=None) == NULL
    for arg, bad in (("ys", MIS), ("rows", ODD), ("places", ODD), ("w", ODD), ("dout", MIS), ("dys", MIS), ("dw", ODD)):
        assert b(**{arg: bad}) == ALIGN
    assert b(T=0, S=0) == OK


def test_gated_act_refusals(L):
    def f(gu=A, type=BF16, S=4, ld=16, F=8, act=0, live=None, h=A, h_ld=8):
        return L.bnn_gated_act(gu, type, S, ld, F, act, live, h, h_ld, None)

    def q(gu=A, type=BF16, S=4, ld=16, F=8, act=0, live=None, h=A, h_ld=128, s=A, s_ld=4):
        return L.bnn_gated_act_f8(gu, type, S, ld, F, act, live, h, h_ld, s, s_ld, None)

    def b(gu=A, type=BF16, S=4, ld=16, F=8, act=0, live=None, h=A, h_ld=8, dgu=A, dgu_ld=16):
        return L.bnn_gated_act_backward(gu, type, S, ld, F, act, live, h, h_ld, dgu, dgu_ld, None)

    for fn in (f, q, b):
        assert fn(S=-1) == fn(F=0) == fn(type=3) == fn(act=4) == fn(act=-1) == SHAPE
        assert fn(ld=15) == fn(h_ld=7) == STRIDE
        assert fn(F=2 ** 28 + 1, ld=2 ** 30, h_ld=2 ** 30) == fn(S=2 ** 31) == UNSUPPORTED
        assert fn(gu=None) == fn(h=None) == NULL and fn(gu=MIS) == fn(h=MIS) == fn(live=A + 2) == ALIGN
        assert fn(S=0, gu=None, h=None) == OK
    assert b(dgu_ld=15) == STRIDE and b(dgu=None) == NULL and b(dgu=MIS) == ALIGN
    assert q(s=None) == NULL and q(s_ld=2) == STRIDE


class _OnTheGpu:
    """What the binding's checks look at of a tensor, without a GPU."""

    def __init__(self, t, device=0):
        self.t, self.device_index, self.is_cuda = t, device, True

    def get_device(self):
        return self.device_index

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_rows_without_room_are_refused():
    """A view whose last row ends with its values, as a slice of whole rows does, has no room for a whole block."""
    q = torch.empty((3, 200), dtype=torch.uint8)
    with pytest.raises(ValueError, match="room for 256"):
        B._padded(q, "q", (3, 200), 256, 16)
    big = torch.empty((3 * 256 - 56,), dtype=torch.uint8)
    with pytest.raises(ValueError, match="last row"):
        B._padded(torch.as_strided(big, (3, 200), (256, 1)), "q", (3, 200), 256, 16)
    fine = B.rows_f8(3, 200, "cpu")
    assert B._padded(fine, "q", (3, 200), 256, 16)[1:] == (256, 768)
    assert B._padded(fine[1:2], "q", (1, 200), 256, 16)[1:] == (256, 256)
    with pytest.raises(ValueError, match="consecutive"):
        B._padded(B.rows_f8(200, 3, "cpu").T, "q", (3, 200), 256, 16)
    with pytest.raises(ValueError, match=r"\[4, 200\] expected"):
        B._padded(fine, "q", (4, 200), 256, 16)


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    t = torch.zeros((4,), dtype=torch.int32)
    assert B._whole(_OnTheGpu(t), "t", torch.int32, 4) == t.data_ptr()
    with pytest.raises(ValueError, match="another device"):
        B._whole(_OnTheGpu(t, 1), "t", torch.int32, 4)
    with pytest.raises(TypeError):
        B._whole(t, "t", torch.int32, 4)
    with pytest.raises(TypeError):
        B._whole(_OnTheGpu(t.long()), "t", torch.int32, 4)
    with pytest.raises(ValueError, match="contiguous"):
        B._whole(_OnTheGpu(torch.zeros((8,), dtype=torch.int32)[::2]), "t", torch.int32, 4)


def test_sizes_reach_every_form_of_the_products():
    from tests import f8_forms as F

    for table, along_k in ((F.PLAIN, False), (F.ROWS, False), (F.ALONG_K, True)):
        for wide, bits16, f, size in F.cases(table):
            assert F.form(*size, wide, bits16, along_k) == f, (size, wide, bits16, along_k)
    for wide, bits16, f, size in F.MANY:
        assert F.form(*size, wide, bits16) == f
    # what the rule can give at all: fp32 scales have no 256 x 256 tiles, none of one a unit, and with fp32 results others are never the fastest
    assert set(F.PLAIN[0, 1]) == set(F.ROWS[0, 1]) == set(F.ALONG_K[0, 1]) == {0, 1, 2, 3, 4, 5, 6, 7, 8, 9}
    assert set(F.PLAIN[0, 0]) == set(F.ROWS[0, 0]) == set(F.ALONG_K[0, 0]) == {0, 2, 3, 5, 6, 7, 8, 9}
    assert set(F.PLAIN[1, 1]) == {1, 2, 3, 5, 6, 7, 9} and set(F.PLAIN[1, 0]) == {1, 3, 6, 7, 9}
    f = B.lib().bnn_testing_f8_form
    assert f(0, 1, 0, 8, 8, 0, 1, 256) == f(8, 0, 0, 8, 8, 0, 1, 256) == f(8, 1, 0, 0, 8, 0, 1, 256) == f(8, 1, 0, 8, 8, 0, 3, 256) == f(8, 1, 0, 8, 8, 0, 1, 0) == -1
