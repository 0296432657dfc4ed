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
    """Up to 4 rows an expert are few; with exact sums (for this call all types but bf16) and 16 MB of weights up to 8, with fp32 scales 12."""
    form = lambda rows, experts, N, K: B.lib().bnn_testing_f8_form(rows, experts, 0, N, K, kind, type, 256)
    most = 4 if type == BF16 else 12 if kind else 8
    for experts, N, K in ((8, 4096, 4096), (1, 16384, 4096), (4, 8192, 512)):  # the last: 16 MB
        assert form(experts * most, experts, N, K) == 9 != form(experts * most + 1, experts, N, K)
    assert form(4 * 4, 4, 8192, 384) == 9 != form(4 * 4 + 1, 4, 8192, 384)
