"""8-bit floating point at its limits: the longest rows, and offsets that no sort gives, with guards around what is written.  Whole numbers,
every sum exact in fp32."""
import pytest
import torch

from paper_1911_04477_amd import binding as B
from tests import f8_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MOST = 2 ** 22 - 128


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def ones_and_zeros(g, rows, K):
    """0 and 1 in e4m3, scales of one; their values."""
    v = torch.randint(0, 2, (rows, R.up(K, 128)), generator=g, device=DEV, dtype=torch.uint8)
    v[:, K:] = 0
    s = torch.full((rows, R.up(R.up(K, 128) // 128, 4)), 127, dtype=torch.uint8, device=DEV)
    return (v * 0x38).view(B.F8)[:, :K], s.view(B.E8M0)[:, : R.up(K, 128) // 128], v[:, :K].float()


def products(a, b):
    """a b^T, some of k at a time: every part and every sum is a whole number below 2^24."""
    return sum(a[:, k: k + 65536] @ b[:, k: k + 65536].T for k in range(0, a.shape[1], 65536))


@pytest.mark.parametrize("M", [3, 270])
@pytest.mark.parametrize("fast", [False, True])
def test_the_longest_rows(M, fast):
    """2^22 - 128 values: sums up to 2^22."""
    print(f"longest {M} fast {fast}", flush=True)
    N = 40
    g = gen(M)
    (qa, sa, a), (qb, sb, b) = ones_and_zeros(g, M, MOST), ones_and_zeros(g, N, MOST)
    want = products(a, b)
    y = B.bnn_linear_f8(qa, sa, qb, sb, dtype=torch.bfloat16 if fast else torch.float32, fast=fast)
    assert torch.equal(y, want.to(y.dtype))
    y = B.bnn_linear_f8(qa, sa, qb, torch.ones((1, MOST // 128), device=DEV), dtype=y.dtype, fast=fast)
    assert torch.equal(y, want.to(y.dtype))
    dw = B.bnn_expert_linear_f8_dw(qa, sa, qb, sb, torch.tensor([0, 128, MOST], dtype=torch.int32, device=DEV), dtype=y.dtype, fast=fast)
    first = a[:, :128] @ b[:, :128].T
    assert torch.equal(dw, torch.stack([first, want - first]).to(y.dtype))


def test_quantised_rows_of_that_length():
    x = torch.randn((2, MOST), generator=gen(5), device=DEV)
    (q, s), (qt, st) = B.bnn_quant_columns_f8(x.T.contiguous()), B.bnn_quant_blocks_f8(x)
    assert torch.equal(q.view(torch.uint8), qt.view(torch.uint8)) and torch.equal(s.view(torch.uint8), st.view(torch.uint8))
    want, p = R.blocks(x[:, -5 * 128:].cpu())
    assert torch.equal(q[:, -5 * 128:].float().cpu().double(), want) and torch.equal(s[:, -5:].view(torch.uint8).cpu().long(), p + 127)


@pytest.mark.parametrize("N,K", [(3, 5), (70, 260), (300, 40)])
@pytest.mark.parametrize("dtype,fast", [(torch.float32, False), (torch.bfloat16, False), (torch.bfloat16, True)])
def test_offsets_of_weight_gradients_outside_the_positions(N, K, dtype, fast):
    """Below 0 and above S they count as these; a group whose end is before its begin is empty.  Nothing around the results is written."""
    S, E = 640, 4
    g = gen(N)
    (qa, sa, a), (qb, sb, b) = ones_and_zeros(g, N, S), ones_and_zeros(g, K, S)
    offsets = torch.tensor([-640, 256, 128, 2 ** 30, 512], dtype=torch.int32, device=DEV)
    room = torch.full((E + 2, N + 2, K + 3), -7.0, dtype=dtype, device=DEV)
    want = room.clone()
    for e, (lo, hi) in enumerate(((0, 256), (256, 256), (128, 640), (640, 640))):
        want[1 + e, :N, :K] = (a[:, lo:hi] @ b[:, lo:hi].T).to(dtype)
    with pytest.raises(B.BnnError):  # off 16 bytes
        B.bnn_expert_linear_f8_dw(qa, sa, qb, sb, offsets, out=room[1: 1 + E, :N, 1: 1 + K], fast=fast)
    flat = torch.full((8 + room.numel(),), -7.0, dtype=dtype, device=DEV)
    start = -(-(N + 2) * (K + 3) // 8) * 8  # the results on 16 bytes, one matrix of room before them
    view = torch.as_strided(flat, (E, N, K), ((N + 2) * (K + 3), K + 3, 1), start)
    B.bnn_expert_linear_f8_dw(qa, sa, qb, sb, offsets, out=view, fast=fast)
    assert torch.equal(view, want[1: 1 + E, :N, :K])
    view.fill_(-7.0)
    assert (flat == -7).all()


@pytest.mark.parametrize("S", [40, 400])
@pytest.mark.parametrize("fast", [False, True])
def test_offsets_of_rows_outside_them(S, fast):
    """The same of rows by expert: rows of one group have its products, rows of none are left alone."""
    N, K = 70, 130
    g = gen(S)
    (qa, sa, a), (qb, sb, b) = ones_and_zeros(g, S, K), ones_and_zeros(g, 4 * N, K)
    offsets = torch.tensor([-5, S // 4, S // 10, S // 2, 7], dtype=torch.int32, device=DEV)
    flat = torch.full(((S + 2) * (N + 2),), -7.0, dtype=torch.bfloat16, device=DEV)
    start = (N + 2 + 7) // 8 * 8
    out = torch.as_strided(flat, (S, N), (N + 2, 1), start)
    B.bnn_expert_linear_f8(qa, sa, offsets, torch.as_strided(qb, (4, N, K), (N * qb.stride(0), qb.stride(0), 1)),
                           torch.as_strided(sb, (4, N, sb.shape[1]), (N * sb.stride(0), sb.stride(0), 1)), out=out, fast=fast)
    w = b.reshape(4, N, K)
    assert torch.equal(out[: S // 10].float(), (a[: S // 10] @ w[0].T).bfloat16().float())
    assert torch.equal(out[S // 4: S // 2].float(), (a[S // 4: S // 2] @ w[2].T).bfloat16().float())
    assert (out[S // 2:] == -7).all()
    out.fill_(-7.0)
    assert (flat == -7).all()
