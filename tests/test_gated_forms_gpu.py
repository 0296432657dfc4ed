"""Every form that the kernels of the 8-bit and gated layers take, each at sizes that reach it (gated_forms.py) and over more steps than
its rings have stages, against the formulas in 64 bits: the bounds of test_gated_layers_gpu.py, inputs that repeat."""
import zlib

import gated_forms
import pytest
import test_gated_layers_gpu as layers
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U32 = 2.0 ** -24


@pytest.fixture(autouse=True)
def inputs_that_repeat(monkeypatch):
    """The same inputs in every process."""
    def gen(*key):
        g = torch.Generator(device=DEV)
        g.manual_seed(zlib.crc32(repr(key).encode()))
        return g

    monkeypatch.setattr(layers, "gen", gen)


def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


PRODUCTS = [(weights, aligned, form, M, N) for (weights, aligned), sizes in gated_forms.PRODUCTS.items() for form, (M, N) in sizes.items()]


def reaches(weights, aligned, form, M, N):
    if units() == gated_forms.UNITS:
        assert gated_forms.product_form(M, N, weights, aligned, units()) == form


# k in bytes: 14 whole steps of 128 and a remainder, the same without one, and fewer whole steps than the deepest ring has stages
@pytest.mark.parametrize("k_bytes", [14 * 128 + 26, 14 * 128, 3 * 128 + 100])
@pytest.mark.parametrize("weights,aligned,form,M,N", PRODUCTS)
def test_products(weights, aligned, form, M, N, k_bytes):
    print(f"product of {weights} weights, form {form}, rows on 16 bytes {aligned}: {M} x {N}, {k_bytes} bytes", flush=True)
    reaches(weights, aligned, form, M, N)
    if weights == 1:
        layers.test_linear_i8(M, N, k_bytes, BF16, True, 16 if aligned else 3)
        return
    gap8 = 16 if aligned else 3
    layers.test_gated_ff_i8(M, k_bytes, N, F32, "gelu", gap8)
    layers.test_gated_ff_i8(M, k_bytes, N, BF16, "silu", gap8)
    K = k_bytes // 2
    gap16 = (-K) % 8 if aligned else (3 if (K + 3) % 8 else 5)
    layers.test_gated_ff(M, K, N, BF16, "silu", gap16)
    layers.test_gated_ff(M, K, N, F16, "gelu_tanh", gap16)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,D,F", gated_forms.BACKWARD)
def test_backward_products(T, D, F, dtype):
    print(f"backward {gated_forms.backward_plan(T, D, F)[:2]}", flush=True)
    layers.test_gated_ff_backward(T, D, F, dtype, "silu", 0)


def many_rows(rows, D, post, pre, gate, vectors, dtype, rtype, gap=0):
    print(f"norm {rows} x {D} {post} {pre} {gate} {dtype} {rtype}", flush=True)
    b, r, s = layers.norm_inputs(layers.gen(rows, D, post, pre), rows, D, dtype, rtype, post, pre, gate, vectors)
    x = layers.norm_parts(b, r, s)
    dr1, dn, _ = layers.norm_bounds(b, r, s, x)
    r1, n = B.bnn_norm_gate(layers.strided(b, gap), layers.strided(r, gap), **s)
    layers.close(r1, x["r1"], layers.rounded(x["r1"], rtype) + dr1, "r'")
    if pre == "none":
        return
    layers.close(n, x["n"], layers.rounded(x["n"], dtype) + dn, "n")
    q, qs = B.rows_i8(rows, D, DEV), torch.empty((rows,), device=DEV)
    again, _ = B.bnn_norm_gate(b, r, q_out=q, q_scale=qs, **s)
    assert torch.equal(again, r1)
    top, worst, step = x["n"].abs().amax(1), dn.amax(1), qs.double()[:, None]
    assert bool(((qs.double() - top / 127).abs() <= worst / 127 + 2 * U32 * top / 127 + layers.TINY[F32]).all())
    layers.close(q.double() * step, x["n"], 0.5 * step + dn + worst[:, None] + 4 * U32 * top[:, None], "q")


# more rows than teams at every number of threads a row: a wave up to 512 values (8192 teams), workgroups of 128 to 512 threads with eight
# values each (4096 to 1024), of 576 to 1024 (768 to 512), the same with sixteen
@pytest.mark.parametrize("post,pre,gate,vectors,dtype,rtype", layers.NORM_KINDS)
@pytest.mark.parametrize("rows,D", [(20000, 5), (20000, 64), (9000, 509), (9000, 1000), (5000, 2321), (2500, 4096), (1600, 4104), (1300, 8192),
                                    (1300, 8191), (1100, 16384), (1100, 10001)])
def test_norm_of_many_rows(rows, D, post, pre, gate, vectors, dtype, rtype):
    many_rows(rows, D, post, pre, gate, vectors, dtype, rtype)


# several rows a team in every form of the backward kernel: waves, workgroups of up to 512 threads with eight values each, of up to 512
# with sixteen (up to 96 KB of vectors in LDS), of up to 1024 with sixteen
@pytest.mark.parametrize("post,pre,gate,vectors,dtype,rtype", layers.NORM_KINDS)
@pytest.mark.parametrize("rows,D", [(20000, 5), (9000, 512), (4000, 1024), (3000, 1023), (700, 4096), (800, 4095), (700, 4104), (600, 6144),
                                    (600, 8192), (600, 8191), (600, 8200), (300, 16384), (600, 16383)])
def test_norm_backward_of_many_rows(rows, D, post, pre, gate, vectors, dtype, rtype):
    layers.test_norm_gate_backward(rows, D, post, pre, gate, vectors, dtype, rtype)


@pytest.mark.parametrize("gate_rows", [2, 100, 257, 1500])
@pytest.mark.parametrize("D", [64, 1000, 4096, 8192])
def test_norm_backward_of_groups(D, gate_rows):
    """Gates of few rows, of a team's rows, of several teams' rows, and a last group cut short."""
    layers.test_norm_gate_backward(2900, D, "rms", "rms", gate_rows, True, BF16, F32)
