"""The longest rows of 8-bit floating point: 2^22 - 128 values, whole blocks at a stride below 2^22.  Every check comes before a launch, no GPU."""
import pytest

from paper_1911_04477_amd import binding as B

OK, NULL, SHAPE, STRIDE, ALIGN, WORKSPACE, HIP, UNSUPPORTED = range(8)
A = 4096  # never read
MOST = 2 ** 22 - 128
LD, S_LD = MOST, 32768


@pytest.mark.parametrize("K,status", [(MOST - 5, NULL), (MOST, NULL), (MOST + 1, UNSUPPORTED), (MOST + 128, UNSUPPORTED)])
@pytest.mark.parametrize("kind", [0, 1])
def test_products(K, status, kind):
    """What is accepted gets as far as the results' pointer, which is NULL; a longer row is refused whatever its stride."""
    L = B.lib()
    for ld in (LD,) if status == NULL else (LD, 2 ** 22, 2 ** 23):
        assert L.bnn_linear_f8(A, ld, A, S_LD, A, ld, A, kind, S_LD, 128, None, 4, 5, K, None, 1, 5, None) == status
        assert L.bnn_expert_linear_f8(A, ld, A, S_LD, A, 2, A, ld, 5 * ld, A, kind, S_LD, S_LD, 128, 4, 5, K, None, 1, 5, None) == status
        assert L.bnn_expert_linear_f8_dw(A, ld, A, S_LD, A, ld, A, S_LD, A, 2, 4, 5, K, None, 1, 5, 20, None) == status


def weight(ld, scale_ld, q=A):
    return B.F8Weight(q, ld, 0, A, scale_ld, 0)


def test_quantisers():
    L = B.lib()

    def f(N, K, out, turned):
        return L.bnn_quant_weight_f8(A + 4, 1, 1, 0, N, K, K, out, turned, None)  # a weight off its alignment: refused last

    long, short = weight(LD, S_LD), weight(128, 4)
    assert f(5, MOST, long, None) == f(MOST, 5, None, long) == f(2 ** 22, 5, short, None) == f(5, 2 ** 22, None, short) == ALIGN
    for more in (MOST + 1, 2 ** 22):
        assert f(5, more, weight(2 ** 22, S_LD), None) == f(more, 5, None, weight(2 ** 22, S_LD)) == UNSUPPORTED
        assert f(5, more, weight(2 ** 22, S_LD), short) == f(more, 5, short, weight(2 ** 22, S_LD)) == UNSUPPORTED
    assert L.bnn_quant_columns_f8(A + 4, 1, 9, 8, A, 1, MOST, 8, A, LD, A, S_LD, None) == ALIGN
    assert L.bnn_quant_columns_f8(A + 4, 1, 9, 8, A, 1, MOST + 1, 8, A, 2 ** 22, A, S_LD, None) == UNSUPPORTED
