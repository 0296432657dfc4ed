"""The choice of sums in 8-bit floating point at the C ABI: bf16 has fast ones, nothing else has.  No launch, no GPU."""
import pytest

from paper_1911_04477_amd import binding as B

NULL, SHAPE = 1, 2
A = 4096  # never read
F32, BF16, F16, FAST = 0, 1, 2, B.FAST_SUMS


@pytest.mark.parametrize("type,status", [(F32, NULL), (BF16, NULL), (F16, NULL), (BF16 | FAST, NULL), (F32 | FAST, SHAPE), (F16 | FAST, SHAPE),
                                         (3 | FAST, SHAPE), (BF16 | 2 * FAST, SHAPE), (BF16 - FAST, SHAPE)])
def test_types_of_results(type, status):
    """With everything else in order but no room for the results."""
    L = B.lib()
    assert L.bnn_linear_f8(A, 256, A, 4, A, 256, A, 0, 4, 1, None, 40, 50, 200, None, type, 50, None) == status
    assert L.bnn_expert_linear_f8(A, 256, A, 4, A, 3, A, 256, 256 * 50, A, 0, 4, 4 * 50, 1, 40, 50, 200, None, type, 50, None) == status
    assert L.bnn_expert_linear_f8_dw(A, 256, A, 4, A, 256, A, 4, A, 3, 40, 50, 200, None, type, 50, 2000, None) == status


@pytest.mark.parametrize("type", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [0, 1])
def test_few_rows(type, kind):
    """Up to 4 rows, on average of the experts, are few; with exact sums (for this call all types but bf16) and 16 MB of weights up to 8, with fp32
    scales 12; of experts, which have uneven rows, 4 and 8."""
    form = lambda rows, experts, N, K: B.lib().bnn_testing_f8_form(rows, experts, 0, N, K, kind, type, 256)
    for experts, N, K, most in ((8, 4096, 4096, (4, 8)), (1, 16384, 4096, (8, 12)), (4, 8192, 512, (4, 8)), (1, 32768, 512, (8, 12)),
                                (4, 8192, 384, (4, 4)), (1, 32768, 384, (4, 4))):  # 16 MB, and less
        n = experts * (4 if type == BF16 else most[kind])
        assert form(n, experts, N, K) == 9 != form(n + 1, experts, N, K)
