"""Sizes whose workgroups hold 2^32 threads and more, which one dimension of a launch does not take: rows of the quantizer, columns of
the 8-bit product with few rows and with tiles."""
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
