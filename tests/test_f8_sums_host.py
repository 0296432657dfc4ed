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
