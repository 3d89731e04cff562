"""Decode attention on inputs whose every step is exact in fp32, so that a row that is missed, taken twice or taken
from another place shows at any length. CPU tensors, 64 bits.

A query holds a single 1, keys are whole numbers from -3 to 0 and the scale is ln 2, which the kernel's log2 e
turns into 1 (their fp32 product rounds to 1): base-2 logits are whole, probabilities 1, 1/2, 1/4 and 1/8 and
every rescaling a power of two. Values are mostly 0 with whole numbers of up to 4 among them: weighted sums are
multiples of 1/8, exact below 2^21 in any order."""
import math

import torch

import cache_ref as ref

SCALE = math.log(2.0)


def pools(gen, G, pages, Hkv, ps, Dh, dtype, token_major=False):
    shape = (G, pages, ps, Hkv, Dh) if token_major else (G, pages, Hkv, ps, Dh)
    k = torch.randint(-3, 1, shape, generator=gen).to(dtype)
    v = torch.randint(1, 5, shape, generator=gen) * (torch.rand(shape, generator=gen) < 1 / 64)
    v = (v * (2 * torch.randint(0, 2, shape, generator=gen) - 1)).to(dtype)
    return (k.transpose(2, 3), v.transpose(2, 3)) if token_major else (k, v)


def queries(gen, R, Hq, Dh, dtype):
    q = torch.zeros(R, Hq, Dh)
    return q.scatter_(2, torch.randint(0, Dh, (R, Hq, 1), generator=gen), 1.0).to(dtype)


def attend(q, kk, vv):
    """q [Hq][Dh] over rows kk, vv [Hkv][n][Dh], all in 64 bits: out [Hq][Dh] and the sum of the weights [Hq]."""
    g = q.shape[0] // kk.shape[0]
    out, total = torch.empty_like(q), torch.empty(q.shape[0], dtype=torch.float64)
    for h in range(kk.shape[0]):
        p = torch.exp2(q[h * g:(h + 1) * g] @ kk[h].t())
        total[h * g:(h + 1) * g] = p.sum(-1)
        out[h * g:(h + 1) * g] = p @ vv[h] / p.sum(-1, keepdim=True)
    return out, total


def decode(q, k, v, table, lens):
    """out and lse and their bounds; k, v one layer [pages][Hkv][page][Dh]."""
    R, Hq, Dh = q.shape
    out, total = torch.zeros((R, Hq, Dh), dtype=torch.float64), torch.zeros((R, Hq), dtype=torch.float64)
    for r in range(R):
        n = int(lens[r])
        if n:
            out[r], total[r] = attend(q[r].double(), ref.rows_of(k, table[r], n), ref.rows_of(v, table[r], n))
    return (out, total.log()) + bounds(out, total, q.dtype)


def bounds(out, total, dtype):
    """Nothing rounds but the division (2 u relative, u = 2^-24), the output's own type, and, in lse, the base-2
    logarithm x = lse / ln 2 (2 u |x|, within a step), the maximum added to it and their product with ln 2, a
    constant within u, each u of the result: under 5 u max(1, |lse|) in all, and 3 u for a maximum below 0."""
    u = 2.0 ** -24
    return (ref.U[dtype] + 2 * u) * out.abs(), u * (3 + 5 * total.log().abs().clamp(min=1.0))
