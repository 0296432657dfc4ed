"""The activations of the gated layers and their slopes, value by value: a projection of one term is that term, so that what
the forward pass saves in fp32 is the function itself.  u is 2^-24."""
import math

import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U32 = 2.0 ** -24


def gelu(z):
    """The normal distribution's function by erfc, which keeps its digits below zero, and its density."""
    t = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return t, torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def saved_of(z, act):
    """act'(z) and act(z) in fp32, and h = act(z) * 1 in the type of z."""
    n = z.numel()
    x = torch.stack([z, torch.ones_like(z)], 1).contiguous()
    wg, wu = (torch.tensor([[a, c]], dtype=z.dtype, device=DEV) for a, c in ((1.0, 0.0), (0.0, 1.0)))
    saved = B.gated_ff_saved(n, 1, DEV)
    h = B.bnn_gated_ff(x, wg, wu, act, saved=saved)
    return saved[0, :, 0], saved[1, :, 0], h[:, 0]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gelu_keeps_its_digits_below_zero(dtype):
    """Every number of the type from -12 to 12 (beyond, exp(-z^2 / 2) leaves fp32's normal numbers): 16 u of the function itself,
    where the function is z times its normal probability, and of the two terms of its slope."""
    bits = torch.arange(1 << 16, device=DEV, dtype=torch.int32).to(torch.int16)
    z = bits.view(dtype)
    z = z[z.float().abs() <= 12]
    slope, value, h = saved_of(z, "gelu")
    t, density = gelu(z.double())
    want = z.double() * t
    off = (value.double() - want).abs()
    bad = ~(off <= 16 * U32 * want.abs() + 2.0 ** -140)
    assert not bool(bad.any()), (z[bad][:4], (off / want.abs())[bad].max() / U32)
    off = (slope.double() - (t + z.double() * density)).abs()
    assert bool((off <= 16 * U32 * (t + (z.double() * density).abs())).all()), float((off / t).max())
    u = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    assert bool(((h.double() - want).abs() <= (u + 16 * U32) * want.abs() + 2.0 ** -25).all())


def test_gelu_in_fp32_from_8_bits():
    """The 8-bit form with fp32 output: projections of one product with scales that are powers of two are exact."""
    for scale in (2.0 ** -4, 2.0 ** -6, 2.0 ** -9):
        x = torch.arange(-128, 128, device=DEV, dtype=torch.int32).to(torch.int8)[:, None].contiguous()
        one, s = torch.ones((1, 1), dtype=torch.int8, device=DEV), torch.full((256,), scale, device=DEV)
        # the second projection is the first: h = act(z) * z
        h = B.bnn_gated_ff_i8(x, s, one, torch.ones(1, device=DEV), one, torch.ones(1, device=DEV), "gelu", dtype=torch.float32)
        z = x[:, 0].double() * scale
        want = z * gelu(z)[0] * z
        assert bool(((h[:, 0].double() - want).abs() <= 17 * U32 * want.abs() + 2.0 ** -140).all()), scale


def test_gelu_at_the_ends():
    """Far out the function is z or 0 and its slope 1 or 0; infinities and NaN as z * (1 + erf(z / sqrt 2)) / 2 has them."""
    z = torch.tensor([14.0, 300.0, 6e4, float("inf"), -14.0, -300.0, -6e4, float("-inf"), float("nan"), 0.0, -0.0], device=DEV).half()
    n = z.numel()
    one = torch.ones((1, 1), dtype=torch.float16, device=DEV)
    saved = B.gated_ff_saved(n, 1, DEV)
    B.bnn_gated_ff(z[:, None].contiguous(), one, one, "gelu", saved=saved)
    value = saved[1, :, 0]
    assert torch.equal(value[:4], z[:4].float()) and bool((value[4:7].abs() < 1e-38).all())
    assert bool(value[7:9].isnan().all()) and bool((value[9:] == 0).all())
    assert torch.equal(saved[0, :3, 0], z[:3].float())  # act'(g) u, with u = z
    assert bool((saved[0, 4:7, 0].abs() < 1e-38).all())
