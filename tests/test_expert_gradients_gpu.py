"""bnn_expert_combine_backward where only one of its results is wanted, which the C ABI allows: the other's pointer and what only that needs are NULL."""
import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def call(ys, rows, places, weights, dout, dys, dweights, S, D):
    p = lambda t: None if t is None else t.data_ptr()
    T, k = places.shape
    st = B.lib().bnn_expert_combine_backward(p(ys), B.FLOATS[dout.dtype], S, D, p(rows), p(places), p(weights), p(dout), D, T, k, D, p(dys), D,
                                             p(dweights), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("D", [3, 40, 512, 513, 2321, 8200])
def test_one_result_alone(D, dtype):
    """The same bits as with both."""
    print(f"alone {D} {dtype}", flush=True)
    T, k, E = 60, 3, 5
    g = gen(D)
    e = torch.randint(-1, E, (T, k), generator=g, device=DEV)
    offsets, rows, places = B.bnn_expert_sort(e, E, 16)
    S = rows.shape[0]
    ys, dout = (torch.randn((n, D), generator=g, device=DEV).to(dtype) for n in (S, T))
    w = torch.rand((T, k), generator=g, device=DEV)
    both = B.bnn_expert_combine_backward(ys, rows, places, w, dout, dys=torch.full((S, D), -7.0, dtype=dtype, device=DEV))
    dys, dw = torch.full((S, D), -7.0, dtype=dtype, device=DEV), torch.full((T, k), -7.0, device=DEV)
    call(None, rows, places, w, dout, dys, None, S, D)
    call(ys, None, places, None, dout, None, dw, S, D)
    assert torch.equal(dys, both[0]) and torch.equal(dw, both[1])


@pytest.mark.parametrize("T,D", [((1 << 20) + 1, 520), ((1 << 22) + 5, 8)])
@pytest.mark.parametrize("given", [False, True])
def test_weights_gradients_of_more_than_2_20_workgroups(T, D, given):
    """One workgroup for a token (D above 512) or four: the grid's last row has workgroups that no token and no row is left for.  rows, not
    needed, may be given all the same, here as positions between experts' rows: there is nothing to clear."""
    print(f"dweights {T} x {D} rows {given}", flush=True)
    S = 3000
    g = gen(T)
    ys = torch.randint(-2, 3, (S, D), generator=g, device=DEV).to(BF16)
    dout = torch.randint(-2, 3, (T, D), generator=g, device=DEV).to(BF16)
    places = torch.randint(-1, S, (T, 1), generator=g, device=DEV, dtype=torch.int32)
    rows = torch.full((S,), -1, dtype=torch.int32, device=DEV) if given else None
    dw = torch.full((T, 1), -7.0, device=DEV)
    call(ys, rows, places, None, dout, None, dw, S, D)
    at = torch.cat([torch.arange(0, T, 997, device=DEV), torch.arange(T - 70, T, device=DEV)])
    p = places[at, 0].long()
    want = torch.where(p >= 0, (ys[p.clamp(min=0)].float() * dout[at].float()).sum(1), 0.0)
    assert torch.equal(dw[at, 0], want) and not (dw == -7).all()


@pytest.mark.parametrize("T,D", [((1 << 20) + 1, 520), ((1 << 22) + 5, 8)])
def test_rows_gradients_of_more_than_2_20_workgroups(T, D):
    """With rows to clear: those named -1 become zeros, others stay."""
    print(f"dys {T} x {D}", flush=True)
    S = 3000
    g = gen(T + 1)
    dout = torch.randn((T, D), generator=g, device=DEV, dtype=BF16)
    places = torch.full((T, 1), -1, dtype=torch.int32, device=DEV)
    rows = torch.where(torch.arange(S, device=DEV) % 3 == 0, -1, -2).to(torch.int32)
    for pos, t in ((1, 0), (2, T - 1), (2998, T // 2)):
        rows[pos], places[t, 0] = t, pos
    dys = torch.full((S, D), -7.0, dtype=BF16, device=DEV)
    call(None, rows, places, None, dout, dys, None, S, D)
    want = torch.full((S, D), -7.0, dtype=BF16, device=DEV)
    want[rows == -1] = 0
    for pos, t in ((1, 0), (2, T - 1), (2998, T // 2)):
        want[pos] = dout[t]
    assert torch.equal(dys, want)
