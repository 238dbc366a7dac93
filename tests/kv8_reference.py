"""Rows held in 8 bits and the attention over them, from their definition in 64 bits (torch, on the CPU)."""
import math

import torch

BLOCK = 32


def exponents(x):
    """x float64 [n][heads][dim], n a multiple of 32 -> int64 [n / 32][heads]: the least e with max|x| <= 448 * 2^e."""
    b = x.reshape(-1, BLOCK, *x.shape[1:]).abs()
    b = torch.where(torch.isfinite(b), b, torch.zeros_like(b))
    most = b.amax(dim=(1, 3))
    e = torch.zeros(most.shape, dtype=torch.int64)
    for i in range(most.shape[0]):
        for h in range(most.shape[1]):
            v = float(most[i, h])
            if v > 0:
                k = -100
                while k < 120 and v > math.ldexp(448.0, k):
                    k += 1
                e[i, h] = k
    return e


def nearest_e4m3(y):
    """float64 -> the nearest e4m3 number, halves to even; beyond 448: 448; not finite: NaN."""
    _, ex = torch.frexp(y.abs().clamp_min(2.0 ** -6))
    step = torch.ldexp(torch.ones_like(y), (ex - 4).to(torch.int32))        # y in [2^(ex-1), 2^ex): 3 bits behind the first
    r = (torch.round(y / step) * step).clamp(-448.0, 448.0)
    return torch.where(torch.isfinite(y), r, torch.full_like(y, float("nan")))


def held(x, e=None, valid=None):
    """What blocks starting at row 0 hold of rows x [n][heads][dim]: float64, same shape. `valid`: rows that count for the exponents
    (default all)."""
    x = x.double()
    n = x.shape[0]
    pad = torch.cat([x, torch.zeros((-n % BLOCK, *x.shape[1:]), dtype=torch.float64)])
    if e is None:
        count = pad.clone()
        if valid is not None:
            count[valid:] = 0
        e = exponents(count)
    unit = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e.to(torch.int32))[:, None, :, None]
    b = pad.reshape(-1, BLOCK, *x.shape[1:])
    return (nearest_e4m3(b / unit) * unit).reshape(pad.shape)[:n]


def attention(q, keys, values, visible):
    """q [T][heads][dim], keys / values [n][heads][dim], visible bool [T][n]; float64. Returns (out, sum p |v|, largest sum |q||k|
    over sqrt(dim) of a visible pair), the last two for bounds."""
    q, keys, values = q.double(), keys.double(), values.double()
    s = torch.einsum("the,nhe->htn", q, keys) / math.sqrt(q.shape[2])
    s = s.masked_fill(~visible[None], float("-inf"))
    p = torch.softmax(s, dim=-1)
    reach = (torch.einsum("the,nhe->htn", q.abs(), keys.abs()) / math.sqrt(q.shape[2])).masked_fill(~visible[None], 0.0)
    return torch.einsum("htn,nhe->the", p, values), torch.einsum("htn,nhe->the", p, values.abs()), float(reach.max())


def attention_bound(out, spread, reach, dim, n):
    """How far a kernel's bfloat16 result may be off. Probabilities are rounded to bfloat16 (2^-8 of each) and so is the result
    (2^-8). Scores are float32 sums of `dim` products (dim + 2 roundings of at most 2^-24 of the sum of magnitudes, `reach`), enter
    exp2 with two more, in the numerator and the denominator: e^(2 d) - 1 < 4 d; exp2 and the float32 sums over n terms add 2^-20
    and n 2^-24."""
    d = (dim + 4) * 2.0 ** -24 * reach
    return 2.0 ** -8 * out.abs() + (1 + 2.0 ** -8) * (2.0 ** -8 + 4 * d + 2.0 ** -20 + 2 * n * 2.0 ** -24) * spread + 1e-30


def ancestors(parent):
    T = len(parent)
    m = torch.zeros(T, T, dtype=torch.bool)
    for i in range(T):
        j = i
        while j >= 0:
            m[i, j] = True
            j = parent[j]
    return m
