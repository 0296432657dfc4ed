"""8-bit floating point and experts on matrices past 2^32 bytes: offsets that pass 32 bits, rows looked at where a wrapped one would land."""
import pytest
import torch

from paper_1911_04477_amd import binding as B
from tests import f8_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def test_quantisers_past_2_32_bytes():
    T, K = 70000, 65536  # 9.2 GB of bf16, 4.6 GB of e4m3
    x = torch.randn((T, K), generator=gen(1), device=DEV, dtype=BF16)
    q, s = B.bnn_quant_blocks_f8(x)
    for lo in (0, 32765, 65533, T - 3):
        want, p = R.blocks(x[lo: lo + 3].cpu())
        assert torch.equal(q[lo: lo + 3].float().cpu().double(), want) and torch.equal(s[lo: lo + 3].view(torch.uint8).cpu().long(), p + 127)
    del q, s
    q, s = B.bnn_quant_columns_f8(x)
    for lo in (0, 30583, 61166, K - 3):
        want, p = R.blocks(x[:, lo: lo + 3].cpu().T)
        assert torch.equal(q[lo: lo + 3].float().cpu().double(), want) and torch.equal(s[lo: lo + 3].view(torch.uint8).cpu().long(), p + 127)
    del q, s
    h = B.bnn_gated_act(x, "relu")
    d = B.bnn_gated_act_backward(x, h, "relu")
    for lo in (0, 32765, 65533, T - 3):
        g, u = x[lo: lo + 3].float().chunk(2, 1)
        assert torch.equal(h[lo: lo + 3], (g.relu() * u).to(BF16))
        hh = h[lo: lo + 3].float()
        assert torch.equal(d[lo: lo + 3], torch.cat([hh * u * (g > 0), hh * g.relu()], 1).to(BF16))


def test_rows_of_experts_past_2_32_bytes():
    T, k, E, D = 40000, 2, 7, 32768
    x = torch.randn((T, D), generator=gen(2), device=DEV, dtype=BF16)
    e = torch.randint(0, E, (T, k), generator=gen(3), device=DEV)
    offsets, rows, places = B.bnn_expert_sort(e, E)
    xs = B.bnn_expert_gather(x, rows, k)
    at = [0, 32767, 32768, 65535, 65536, T * k - 1]
    assert torch.equal(xs[at], x[rows[at].long() // k])
    out = B.bnn_expert_combine(xs, places)
    assert torch.equal(out[[0, 16384, T - 1]], (2 * x[[0, 16384, T - 1]].float()).to(BF16))
    dys, dw = B.bnn_expert_combine_backward(xs, rows, places, None, x)
    assert torch.equal(dys[at], x[rows[at].long() // k])
    norms = x[[0, 16384, T - 1]].double().square().sum(1)
    assert ((dw[[0, 16384, T - 1]].double() - norms[:, None]).abs() <= D * 2.0 ** -24 * norms[:, None]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_products_past_2_32_bytes(dtype):
    """Results and operands past 2^32 bytes; whole numbers, so that every result is exact."""
    M, N, K = 70000, 33000, 200
    a = torch.randint(-4, 5, (M, K), generator=gen(4), device=DEV).float()
    b = torch.randint(-4, 5, (N, K), generator=gen(5), device=DEV).float()
    y = B.bnn_linear_f8(*B.bnn_quant_blocks_f8(a), *B.bnn_quant_weight_f8(b, turned=False)[0], dtype=dtype)
    for lo in (0, 32500, 65070, M - 5):
        assert torch.equal(y[lo: lo + 5], (a[lo: lo + 5] @ b.T).to(dtype))
    del y
    E, S, N, K = 5, 40, 16500, 66000  # 5.4 GB of weights
    offsets = torch.tensor([0, 9, 9, 20, 30, S], dtype=torch.int32, device=DEV)
    w = torch.empty((E, N, R.up(K, 128)), dtype=torch.uint8, device=DEV).zero_()
    for e in range(E):
        w[e, :, :K] = torch.randint(0, 2, (N, K), generator=gen(6 + e), device=DEV, dtype=torch.uint8) * 0x38  # 0 or 1.0
    s = torch.full((E, R.up(N, 128) // 128, R.up(R.up(K, 128) // 128, 4)), 127, dtype=torch.uint8, device=DEV)
    x = torch.randint(-2, 3, (S, K), generator=gen(20), device=DEV).float()
    y = B.bnn_expert_linear_f8(*B.bnn_quant_blocks_f8(x), offsets, w.view(B.F8)[..., :K], s.view(B.E8M0)[..., : R.up(K, 128) // 128], dtype=dtype)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi > lo:
            at = torch.tensor([0, 1, 8000, N - 1], device=DEV)
            want = x[lo:hi] @ (w[e, at, :K].float() / 0x38).T
            assert torch.equal(y[lo:hi][:, at], want.to(dtype)), e
