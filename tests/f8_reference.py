"""Definitions of 8-bit floating point with block scales and of the expert layers, in 64 bits on the CPU, and inputs for their tests."""
import torch

from paper_1911_04477_amd import binding as B

BLOCK = 128
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def up(n, to):
    return (n + to - 1) // to * to


def e4m3(v):
    """The nearest e4m3 value to a float64 tensor of magnitudes up to 448, ties to even; NaN and infinities are NaN."""
    _, e = torch.frexp(v)
    step = torch.pow(torch.tensor(2.0, dtype=torch.float64), ((e - 1).clamp(min=-6) - 3).double())
    r = torch.round(v / step) * step
    return torch.where(torch.isfinite(v), r, torch.full_like(v, float("nan")))


def exponent(top):
    """The least whole p >= -100 with top <= 448 * 2^p."""
    p = torch.full(top.shape, -100, dtype=torch.int64)
    m, e = torch.frexp(top / 448.0)
    p = torch.where(top > 0, torch.where(m == 0.5, e - 1, e).long(), p)
    return p.clamp(min=-100)


def power(p):
    return torch.pow(torch.tensor(2.0, dtype=torch.float64), p.double())


def blocks(x):
    """(values of rows / 2^p in e4m3, p [rows, blocks]) of a matrix on the CPU."""
    x = x.double()
    rows, K = x.shape
    b = torch.nn.functional.pad(x, (0, up(K, BLOCK) - K)).reshape(rows, -1, BLOCK)
    p = exponent(torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax(2))
    return e4m3(b / power(p)[..., None]).reshape(rows, -1)[:, :K], p


def values(q, p):
    return q * power(p).repeat_interleave(BLOCK, 1)[:, : q.shape[1]]


def weight(w):
    """(q [N, K], p [blocks of N, blocks of K])."""
    w = w.double()
    N, K = w.shape
    b = torch.nn.functional.pad(w, (0, up(K, BLOCK) - K, 0, up(N, BLOCK) - N)).reshape(up(N, BLOCK) // BLOCK, BLOCK, -1, BLOCK)
    p = exponent(torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax((1, 3)))
    return e4m3(b / power(p)[:, None, :, None]).reshape(up(N, BLOCK), -1)[:N, :K], p


def weight_values(q, p):
    return q * power(p).repeat_interleave(BLOCK, 0)[: q.shape[0]].repeat_interleave(BLOCK, 1)[:, : q.shape[1]]


def sort(experts, E, align, S):
    """offsets, rows, places by going through the slots one after the other."""
    flat = experts.reshape(-1).tolist()
    slots = [[i for i, e in enumerate(flat) if e == x] for x in range(E)] if len(flat) * E < 1 << 22 else None
    if slots is None:
        slots = [[] for _ in range(E)]
        for i, e in enumerate(flat):
            if 0 <= e < E:
                slots[e].append(i)
    offsets, rows, places = [0], [-2] * S, [-1] * len(flat)
    for mine in slots:
        at = offsets[-1]
        end = at + up(len(mine), align)
        for i in range(at, end):
            rows[i] = -1
        for i, s in enumerate(mine):
            rows[at + i], places[s] = s, at + i
        offsets.append(end)
    as_int = dict(dtype=torch.int32)
    return torch.tensor(offsets, **as_int), torch.tensor(rows, **as_int), torch.tensor(places, **as_int).reshape(experts.shape)


def act(z, name):
    """An activation and its derivative in 64 bits."""
    if name == "silu":
        t = torch.sigmoid(z)
        return z * t, t * (1 + z * (1 - t))
    if name == "gelu":
        c = 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)
        return z * c, c + z * torch.exp(-z * z / 2) * (0.5 / torch.pi) ** 0.5
    if name == "gelu_tanh":
        k = (2 / torch.pi) ** 0.5
        t = torch.sigmoid(2 * k * (z + 0.044715 * z ** 3))
        return z * t, t + z * t * (1 - t) * 2 * k * (1 + 3 * 0.044715 * z * z)
    return torch.relu(z), (z > 0).double()


def stored(q, p, dev="cuda:0", share=False):
    """q, p (of the functions above) as the tensors that the products take: rows with room for whole blocks, NaN behind the scales."""
    lead = q.shape[:-1]
    K = q.shape[-1]
    buf = torch.zeros((*lead, up(K, BLOCK)), dtype=torch.uint8)
    buf[..., :K] = q.to(torch.float32).to(B.F8).view(torch.uint8)
    s = torch.full((*p.shape[:-1], up(p.shape[-1], 4)), 255, dtype=torch.uint8)
    s[..., : p.shape[-1]] = (p + 127).to(torch.uint8)
    return buf.to(dev).view(B.F8)[..., :K], s.to(dev).view(B.E8M0)[..., : p.shape[-1]]


def whole_numbers(g, rows, K, scale_rows=None):
    """(q, p) of small whole numbers and scales 1, 2 and 4: every sum of products of two such matrices is exact in fp32."""
    q = torch.randint(-4, 5, (rows, K), generator=g).double()
    p = torch.randint(0, 3, (rows if scale_rows is None else scale_rows, up(K, BLOCK) // BLOCK), generator=g)
    return q, p
