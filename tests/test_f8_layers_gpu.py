"""8-bit floating point with block scales: the quantisers bit for bit against their definition, the products exactly on whole numbers
(every sum is exact in fp32, so any wrong row, block or scale shows) and within a derived bound on others."""
import pytest
import torch

from paper_1911_04477_amd import binding as B
from tests import f8_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


def gen(*key):
    g = torch.Generator()
    g.manual_seed(sum((i + 1) * 7919 * int(k) for i, k in enumerate(key)) % (1 << 31))
    return g


def strided(x, gap):
    """On the GPU, in rows that are `gap` elements longer, NaN between them."""
    big = torch.full((x.shape[0], x.shape[1] + gap), float("nan"), dtype=x.dtype)
    big[:, : x.shape[1]] = x
    return big.to(DEV)[:, : x.shape[1]]


def bytes_of(t):
    return t.contiguous().view(torch.uint8).cpu()


def check_rows(q, scale, want_q, want_p, name=""):
    """Stored rows against (q, p) of the reference: values, scales, and zeros behind the last value."""
    got = q.float().cpu().double()
    bad = ~((got == want_q) | (got.isnan() & want_q.isnan()))
    assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][:3], want_q[bad][:3])
    assert torch.equal(bytes_of(scale).long(), want_p + 127), name
    rows, K = q.shape
    whole = torch.as_strided(q.view(torch.uint8), (rows, R.up(K, 128)), (q.stride(0), 1), q.storage_offset())
    assert not whole[:, K:].any(), name


def awkward(g, rows, K):
    """Normal rows over many magnitudes, with zeros, ties between two e4m3 values and the ends of the range."""
    x = torch.randn((rows, K), generator=g) * torch.pow(torch.tensor(2.0), torch.randint(-20, 20, (rows, 1), generator=g).float())
    pick = torch.randint(0, 12, (rows, K), generator=g)
    x = torch.where(pick == 0, torch.zeros(()), x)
    x = torch.where(pick == 1, torch.tensor(1.0625), x)       # between 1 and 1.125
    x = torch.where(pick == 2, torch.tensor(-1.1875), x)
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K,gap", [(1, 1, 0), (3, 5, 0), (5, 7, 1), (2, 8, 0), (9, 127, 0), (4, 128, 3), (3, 129, 0), (33, 300, 4), (7, 512, 0),
                                        (5, 2321, 0), (257, 1024, 0), (2, 16384, 8)])
def test_quant_blocks(rows, K, gap, dtype):
    print(f"blocks {rows} x {K} gap {gap} {dtype}", flush=True)
    x = awkward(gen(rows, K, gap), rows, K).to(dtype)
    q, s = B.rows_f8(rows, K, DEV), B.scales_f8(rows, K, DEV)
    torch.as_strided(q.view(torch.uint8), (rows, q.stride(0)), (q.stride(0), 1)).fill_(77)
    B.bnn_quant_blocks_f8(strided(x, gap), q, s)
    check_rows(q, s, *R.blocks(x))


@pytest.mark.parametrize("dtype", TYPES)
def test_quant_blocks_every_value_and_the_ends(dtype):
    """Every 16-bit value (fp32: those of bf16) in blocks of its own kind, and beside infinities and NaN."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(F16 if dtype == F16 else BF16).to(dtype).reshape(512, 128)
    q, s = B.bnn_quant_blocks_f8(x.to(DEV))
    check_rows(q, s, *R.blocks(x))
    x = torch.randn((6, 256), generator=gen(1)).to(dtype)
    x[0, 3], x[1, 130], x[2, 7], x[3] = float("inf"), float("-inf"), float("nan"), 0.0
    x[4] = torch.finfo(dtype).max
    x[5] = torch.finfo(dtype).tiny
    q, s = B.bnn_quant_blocks_f8(x.to(DEV))
    check_rows(q, s, *R.blocks(x))


@pytest.mark.parametrize("K", [5, 200, 1024])
def test_quant_blocks_of_slots(K):
    T, k = 9, 3
    x = torch.randn((T, K), generator=gen(K)).to(BF16)
    rows = torch.tensor([4, -1, 26, -2, 0, 27, 13, -7, 2 ** 31 - 1, 13, -1], dtype=torch.int32)
    S = rows.numel()
    q, s = B.rows_f8(S, K, DEV), B.scales_f8(S, K, DEV)
    q.view(torch.uint8).fill_(9)
    s.view(torch.uint8).fill_(9)
    B.bnn_quant_blocks_f8(x.to(DEV), q, s, rows=rows.to(DEV), k=k)
    want, p = R.blocks(x)
    for i, r in enumerate(rows.tolist()):
        if 0 <= r < T * k:
            check_rows(q[i: i + 1], s[i: i + 1], want[r // k][None], p[r // k][None], i)
        elif r == -1:
            check_rows(q[i: i + 1], s[i: i + 1], torch.zeros((1, K)), torch.full((1, p.shape[1]), -100), i)
        else:
            assert (bytes_of(q[i]) == 9).all() and (bytes_of(s[i]) == 9).all(), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D,gap", [(1, 1, 0), (1, 64, 0), (5, 7, 2), (127, 63, 0), (128, 65, 0), (129, 200, 1), (300, 513, 0), (1000, 72, 8)])
def test_quant_columns(T, D, gap, dtype):
    print(f"columns {T} x {D} gap {gap} {dtype}", flush=True)
    x = awkward(gen(T, D, gap), T, D).to(dtype)
    x[0, 0] = float("inf") if T > 3 else 1.0
    q, s = B.bnn_quant_columns_f8(strided(x, gap))
    check_rows(q, s, *R.blocks(x.T))


def test_quant_columns_of_slots():
    T, k, D = 50, 2, 130
    x = torch.randn((T, D), generator=gen(5)).to(F16)
    rows = torch.randint(-2, T * k + 1, (333,), generator=gen(6)).to(torch.int32)
    q, s = B.bnn_quant_columns_f8(x.to(DEV), rows=rows.to(DEV), k=k)
    r = rows.long()
    picked = torch.where(((r >= 0) & (r < T * k))[:, None], x[(r // k).clamp(0, T - 1)], torch.zeros((), dtype=F16))
    check_rows(q, s, *R.blocks(picked.T))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,N,K", [(None, 1, 1), (None, 5, 7), (None, 128, 128), (None, 129, 127), (3, 200, 300), (2, 64, 515), (None, 1000, 264)])
def test_quant_weight(E, N, K, dtype):
    print(f"weight {E} x {N} x {K} {dtype}", flush=True)
    w = torch.stack([awkward(gen(N, K, i), N, K) for i in range(E or 1)]).to(dtype)
    w[0, N // 2, K // 2] = float("nan")
    (q, s), (qt, st) = B.bnn_quant_weight_f8(w.to(DEV) if E else w[0].to(DEV))
    alone, none = B.bnn_quant_weight_f8(w.to(DEV) if E else w[0].to(DEV), turned=False)
    assert none is None and torch.equal(bytes_of(alone[0]), bytes_of(q)) and torch.equal(bytes_of(alone[1]), bytes_of(s))
    for e in range(E or 1):
        want, p = R.weight(w[e])
        parts = (q[e], s[e], qt[e], st[e]) if E else (q, s, qt, st)
        check_rows(parts[0], parts[0].new_zeros((N, 1)).view(torch.uint8), want, torch.full((N, 1), -127))
        assert torch.equal(bytes_of(parts[1]).long(), p + 127)
        check_rows(parts[2], parts[2].new_zeros((K, 1)).view(torch.uint8), want.T, torch.full((K, 1), -127))
        assert torch.equal(bytes_of(parts[3]).long(), p.T + 127)


def scales_of(g, kind, N, K):
    """(scales as the product takes them, [N, blocks] of their values): a row each, a row for 128, or fp32 for 128."""
    blocks, n = R.up(K, 128) // 128, R.up(N, 128) // 128
    if kind == "f32":
        s = torch.randint(-5, 6, (n, blocks), generator=g).double()
        return s.float().to(DEV), s.repeat_interleave(128, 0)[:N]
    p = torch.randint(0, 3, (N if kind == "row" else n, blocks), generator=g)
    _, s = R.stored(torch.zeros((p.shape[0], K)), p)
    return s, R.power(p if kind == "row" else p.repeat_interleave(128, 0)[:N])


# rows by columns of every form of the products, with edges in the middle of tiles, and depths of one block to many
SIZES = [(1, 1, 1), (1, 64, 128), (3, 17, 300), (16, 130, 129), (16, 256, 4096 + 5), (17, 33, 640), (33, 70, 257), (64, 200, 1000), (100, 4096, 384),
         (257, 300, 900), (500, 2321, 520), (1000, 3001, 650), (2049, 4100, 385), (4096, 4096, 130)]


@pytest.mark.parametrize("kind", ["row", "block", "f32"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_exact(M, N, K, kind):
    print(f"linear {M} x {N} x {K} {kind}", flush=True)
    g = gen(M, N, K)
    a, pa = R.whole_numbers(g, M, K)
    b = torch.randint(-4, 5, (N, K), generator=g).double()
    sb, vb = scales_of(g, kind, N, K)
    qa, sa = R.stored(a, pa)
    qb, _ = R.stored(b, torch.zeros((N, 1), dtype=torch.int64))
    want = R.values(a, pa).float().to(DEV) @ (b * vb.repeat_interleave(128, 1)[:, :K]).float().to(DEV).T  # exact: whole numbers below 2^24
    room = torch.full((M, N + 3), -7.0, device=DEV)
    got = B.bnn_linear_f8(qa, sa, qb, sb, out=room[:, :N])
    assert torch.equal(got, want)
    assert (room[:, N:] == -7).all()
    bias = torch.randint(-9, 10, (N,), generator=g).float().to(DEV)
    assert torch.equal(B.bnn_linear_f8(qa, sa, qb, sb, bias, dtype=F32), want + bias)
    assert torch.equal(B.bnn_linear_f8(qa, sa, qb, sb, bias), (want + bias).to(BF16))
    assert torch.equal(B.bnn_linear_f8(qa, sa, qb, sb, dtype=F16), want.to(F16))


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (64, 384, 2321), (300, 513, 1000)])
@pytest.mark.parametrize("wide", [False, True])
def test_linear_of_quantised_rows(M, N, K, wide):
    """y from x and w: what the stored values give, up to the sums' roundings.  A sum of K products in fp32, however its adder
    drops bits below the last, is off by at most K * 2^-23 of the sum of magnitudes, the scales' and the result's rounding by 3 * 2^-24."""
    g = gen(M, N, K)
    x, w = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g) / K ** 0.5
    q, s = B.bnn_quant_blocks_f8(x.to(DEV))
    a, b = R.values(*R.blocks(x)), None
    if wide:
        top = torch.nn.functional.pad(w, (0, R.up(K, 128) - K, 0, R.up(N, 128) - N)).reshape(R.up(N, 128) // 128, 128, -1, 128).abs().amax((1, 3))
        sw = (top / 448).contiguous()
        full = sw.repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        v = (w / full).to(B.F8)
        b = v.double() * full.double()
        y = B.bnn_linear_f8(q, s, R.stored(v.double(), torch.zeros((N, 1), dtype=torch.int64))[0], sw.to(DEV), dtype=F32)
    else:
        wq, _ = B.bnn_quant_weight_f8(w.to(DEV), turned=False)
        b = R.weight_values(*R.weight(w))
        y = B.bnn_linear_f8(q, s, *wq, dtype=F32)
    want, sums = (a.to(DEV) @ b.to(DEV).T), (a.abs().to(DEV) @ b.abs().to(DEV).T)
    assert ((y.double() - want).abs() <= (K * 2.0 ** -23 + 3 * 2.0 ** -24) * sums).all()


def test_training_step_of_a_linear_layer():
    """y, dx and dw from bf16 tensors against products of the reference's quantised values, within the bound above."""
    M, N, K = 300, 200, 264
    g = gen(7)
    x, w, dy = (torch.randn(s, generator=g).to(BF16) for s in ((M, K), (N, K), (M, N)))
    (wq, wt), X = B.bnn_quant_weight_f8(w.to(DEV)), x.to(DEV)
    y = B.bnn_linear_f8(*B.bnn_quant_blocks_f8(X), *wq, dtype=F32)
    dx = B.bnn_linear_f8(*B.bnn_quant_blocks_f8(dy.to(DEV)), *wt, dtype=F32)
    dw = B.bnn_linear_f8(*B.bnn_quant_columns_f8(dy.to(DEV)), *B.bnn_quant_columns_f8(X), dtype=F32)
    W = R.weight_values(*R.weight(w))
    for got, a, b in ((y, R.values(*R.blocks(x)), W.T), (dx, R.values(*R.blocks(dy)), W),
                      (dw, R.values(*R.blocks(dy.T)), R.values(*R.blocks(x.T)).T)):
        n = a.shape[1]
        assert ((got.cpu().double() - a @ b).abs() <= (n * 2.0 ** -23 + 2.0 ** -24) * (a.abs() @ b.abs())).all()


def test_gradients_against_differences():
    """The loss of y's definition is linear in x and in w where their quantised values are: a step of a whole unit in one value, inputs
    whole numbers that e4m3 holds, changes it by that value's gradient exactly."""
    M, N, K = 5, 6, 140
    g = gen(11)
    x, w, c = (torch.randint(-3, 4, s, generator=g).float() for s in ((M, K), (N, K), (M, N)))

    def loss(x, w):
        wq, _ = B.bnn_quant_weight_f8(w.to(DEV), turned=False)
        return float((B.bnn_linear_f8(*B.bnn_quant_blocks_f8(x.to(DEV)), *wq, dtype=F32).double() * c.to(DEV)).sum())

    _, wt = B.bnn_quant_weight_f8(w.to(DEV), plain=False)
    dx = B.bnn_linear_f8(*B.bnn_quant_blocks_f8(c.to(DEV)), *wt, dtype=F32)
    dw = B.bnn_linear_f8(*B.bnn_quant_columns_f8(c.to(DEV)), *B.bnn_quant_columns_f8(x.to(DEV)), dtype=F32)
    at = loss(x, w)
    for i, k in ((0, 0), (4, 139), (2, 128)):
        moved = x.clone()
        moved[i, k] += 1
        assert loss(moved, w) - at == float(dx[i, k])
        moved = w.clone()
        moved[i, k] += 1
        assert loss(x, moved) - at == float(dw[i, k])


def test_values_that_are_not_numbers_reach_their_results_only():
    M, N, K = 20, 40, 300
    g = gen(3)
    x, w = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g)
    x[3, 5], x[9, 299], w[7, 1] = float("nan"), float("inf"), float("-inf")
    wq, _ = B.bnn_quant_weight_f8(w.to(DEV), turned=False)
    y = B.bnn_linear_f8(*B.bnn_quant_blocks_f8(x.to(DEV)), *wq, dtype=F32).cpu()
    nan = torch.zeros((M, N), dtype=torch.bool)
    nan[3], nan[9], nan[:, 7] = True, True, True
    assert torch.equal(y.isnan(), nan)


def test_range_of_scales():
    """Scales at both ends: sums that pass fp32's range are infinite, those below it zero, and nothing else is."""
    for p in (-100, -60, 0, 60, 100, 120):
        a, _ = R.stored(torch.full((2, 128), 448.0, dtype=torch.float64), torch.zeros((2, 1), dtype=torch.int64))
        _, s = R.stored(torch.zeros((2, 128)), torch.full((2, 1), p, dtype=torch.int64))
        y = B.bnn_linear_f8(a, s, a, s, dtype=F32).cpu().double()
        want = 448.0 ** 2 * 128 * 2.0 ** (2 * p)
        if want > 3.4e38:
            assert y.isinf().all()
        elif want < 1e-37:
            assert (y <= want).all() and (y >= 0).all()
        else:
            assert (y == want).all()


# ---- experts' products ----------------------------------------------------------------------------------------------
COUNTS = [[1], [0, 0, 5], [16, 0, 1, 17], [3] * 8, [0, 130, 257, 0, 1], [40, 25, 31, 90, 8, 0, 64, 64], [1] * 70 + [0] * 10 + [5, 0, 300], [700, 900, 3],
          [0] * 4]


@pytest.mark.parametrize("kind", ["row", "block", "f32"])
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}_{sum(c)}")
@pytest.mark.parametrize("N,K", [(1, 5), (200, 384), (515, 257)])
def test_expert_linear_exact(counts, N, K, kind):
    print(f"experts {counts} {N} x {K} {kind}", flush=True)
    E, S = len(counts), sum(counts) + 3
    g = gen(E, S, N)
    offsets = torch.tensor([0] + counts, dtype=torch.int64).cumsum(0).to(torch.int32)
    a, pa = R.whole_numbers(g, S, K)
    b = torch.randint(-4, 5, (E, N, K), generator=g).double()
    made = [scales_of(g, kind, N, K) for _ in range(E)]
    if kind == "f32":
        sb = torch.stack([s for s, _ in made])
    else:
        sb = torch.stack([torch.as_strided(s.view(torch.uint8), (s.shape[0], s.stride(0)), (s.stride(0), 1)) for s, _ in made]).view(B.E8M0)[..., : R.up(K, 128) // 128]
    qa, sa = R.stored(a, pa)
    qb, _ = R.stored(b, torch.zeros((E, N, 1), dtype=torch.int64))
    want = torch.full((S, N), -7.0, dtype=torch.float64)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        want[lo:hi] = R.values(a, pa)[lo:hi] @ (b[e] * made[e][1].repeat_interleave(128, 1)[:, :K]).T
    for dtype in (F32, BF16):
        out = torch.full((S, N), -7.0, dtype=dtype, device=DEV)
        got = B.bnn_expert_linear_f8(qa, sa, offsets.to(DEV), qb, sb, out=out)
        assert torch.equal(got.cpu(), want.float().to(dtype)), dtype


@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [1, 2, 0, 3], [5, 0, 9, 1]], ids=str)
@pytest.mark.parametrize("N,K", [(1, 1), (5, 300), (200, 130), (513, 700)])
def test_expert_weight_gradients_exact(counts, N, K):
    print(f"dw {counts} {N} x {K}", flush=True)
    E, S = len(counts), sum(counts) * 128 + 70  # positions behind the last group hold NaN
    g = gen(E, S, N, K)
    offsets = torch.tensor([0] + counts, dtype=torch.int64).cumsum(0) * 128
    (a, pa), (b, pb) = R.whole_numbers(g, N, S), R.whole_numbers(g, K, S)
    want = torch.stack([R.values(a, pa)[:, lo:hi] @ R.values(b, pb)[:, lo:hi].T for lo, hi in zip(offsets[:-1], offsets[1:])])
    a[:, int(offsets[-1]):], b[:, int(offsets[-1]):] = float("nan"), float("nan")
    got = B.bnn_expert_linear_f8_dw(*R.stored(a, pa), *R.stored(b, pb), offsets.to(torch.int32).to(DEV))
    assert torch.equal(got.cpu().double(), want)
    room = torch.full((E, N + 1, K + 2), -7.0, dtype=BF16, device=DEV)
    B.bnn_expert_linear_f8_dw(*R.stored(a, pa), *R.stored(b, pb), offsets.to(torch.int32).to(DEV), out=room[:, :N, :K])
    assert torch.equal(room[:, :N, :K].cpu(), want.float().to(BF16))
    assert (room[:, N:] == -7).all() and (room[:, :, K:] == -7).all()


def test_offsets_out_of_range_stay_inside():
    """Offsets count as 0 or S where they are outside, and never go down: nothing outside the rows is read or written."""
    S, N, K, E = 40, 64, 128, 4
    a, pa = R.whole_numbers(gen(2), S, K)
    b = torch.randint(-4, 5, (E, N, K), generator=gen(3)).double()
    qb, sb = R.stored(b, torch.zeros((E, 1, 1), dtype=torch.int64))
    offsets = torch.tensor([-5, 10, 4, 2 ** 30, 7], dtype=torch.int32)
    out = torch.full((S, N), -7.0, device=DEV)
    B.bnn_expert_linear_f8(*R.stored(a, pa), offsets.to(DEV), qb, sb, out=out)
    v = R.values(a, pa)
    assert torch.equal(out[:4].cpu().double(), v[:4] @ b[0].T)
    dw = B.bnn_expert_linear_f8_dw(*R.stored(a.T.contiguous(), torch.zeros((K, 1), dtype=torch.int64)), *R.stored(a.T.contiguous(), torch.zeros((K, 1), dtype=torch.int64)),
                                   (offsets * 128).to(DEV))
    assert dw.shape == (E, K, K)


# ---- every kernel form ------------------------------------------------------------------------------------------------
from tests import f8_forms as F  # noqa: E402


def whole_on_gpu(g, rows, K, scale_rows=None):
    """Whole numbers with scales 1, 2 and 4 for rows, or for 128 of them, made on the GPU: (stored q, stored scales, values in fp32)."""
    blocks = R.up(K, 128) // 128
    q = torch.randint(-4, 5, (rows, K), generator=g, device=DEV).float()
    p = torch.randint(0, 3, (scale_rows or rows, blocks), generator=g, device=DEV)
    stored = B.rows_f8(rows, K, DEV)
    torch.as_strided(stored.view(torch.uint8), (rows, stored.stride(0)), (stored.stride(0), 1)).zero_()
    stored.copy_(q.to(B.F8))
    s = B.scales_f8(scale_rows or rows, K, DEV)
    s.view(torch.uint8).copy_((p + 127).to(torch.uint8))
    each = p if scale_rows is None else p.repeat_interleave(128, 0)[:rows]
    return stored, s, q * torch.pow(2.0, each.float()).repeat_interleave(128, 1)[:, :K]


def gpu_gen(*key):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum((i + 1) * 7919 * int(k) for i, k in enumerate(key)) % (1 << 31))
    return g


def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("wide,bits16,form,size", F.cases(F.PLAIN), ids=str)
def test_every_form_plain(wide, bits16, form, size):
    print(f"form {form} wide {wide} bits16 {bits16} {size}", flush=True)
    assert units() == 256  # the sizes are for this many
    _, M, N, K = size
    g = gpu_gen(M, N, K)
    qa, sa, a = whole_on_gpu(g, M, K)
    qb, sb, b = whole_on_gpu(g, N, K, None if not wide else R.up(N, 128) // 128)
    if wide:
        sb = sb.float().contiguous()
    want = a @ b.T
    bias = torch.randint(-9, 10, (N,), generator=g, device=DEV).float()
    for dtype in ((BF16, F16) if bits16 else (F32,)):
        room = torch.full((M, N + 1), -7.0, dtype=dtype, device=DEV)
        assert torch.equal(B.bnn_linear_f8(qa, sa, qb, sb, bias, out=room[:, :N]), (want + bias).to(dtype))
        assert (room[:, N:] == -7).all()


@pytest.mark.parametrize("wide,bits16,form,size", F.cases(F.ROWS) + F.MANY, ids=str)
def test_every_form_of_rows_by_expert(wide, bits16, form, size):
    print(f"form {form} wide {wide} bits16 {bits16} {size}", flush=True)
    E, S, N, K = size
    g = gpu_gen(E, S, N, K)
    cuts = torch.randint(0, S - 4, (E - 1,), generator=g, device=DEV).sort().values.tolist()
    bounds = [0, *cuts, S - 5]  # five rows behind the last expert's
    offsets = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    qa, sa, a = whole_on_gpu(g, S, K)
    qb, sb, b = whole_on_gpu(g, E * R.up(N, 128), K, None if not wide else E * R.up(N, 128) // 128)
    qb = torch.as_strided(qb, (E, N, K), (R.up(N, 128) * qb.stride(0), qb.stride(0), 1))
    b = b.reshape(E, -1, K)[:, :N]
    sb = sb.float().contiguous().reshape(E, -1, sb.shape[1]) if wide else torch.as_strided(sb, (E, N, sb.shape[1]), (R.up(N, 128) * sb.stride(0), sb.stride(0), 1))
    dtype = BF16 if bits16 else F32
    want = torch.full((S, N), -7.0, dtype=dtype, device=DEV)
    for e in range(E):
        want[bounds[e]: bounds[e + 1]] = (a[bounds[e]: bounds[e + 1]] @ b[e].T).to(dtype)
    got = B.bnn_expert_linear_f8(qa, sa, offsets, qb, sb, out=torch.full((S, N), -7.0, dtype=dtype, device=DEV))
    assert torch.equal(got, want)


@pytest.mark.parametrize("wide,bits16,form,size", F.cases(F.ALONG_K), ids=str)
def test_every_form_of_weight_gradients(wide, bits16, form, size):
    print(f"form {form} bits16 {bits16} {size}", flush=True)
    E, N, K, k = size
    blocks = E * (k // 128) - 1  # of all groups: the rule has k for their mean, rounded up
    g = gpu_gen(E, N, K, k)
    cuts = torch.randint(0, blocks + 1, (E - 1,), generator=g, device=DEV).sort().values.tolist()
    bounds = [0, *[128 * c for c in cuts], 128 * blocks]
    S = 128 * blocks
    qa, sa, a = whole_on_gpu(g, N, S)
    qb, sb, b = whole_on_gpu(g, K, S)
    dtype = BF16 if bits16 else F32
    got = B.bnn_expert_linear_f8_dw(qa, sa, qb, sb, torch.tensor(bounds, dtype=torch.int32, device=DEV), dtype=dtype)
    for e in range(E):
        assert torch.equal(got[e], (a[:, bounds[e]: bounds[e + 1]] @ b[:, bounds[e]: bounds[e + 1]].T).to(dtype)), e
