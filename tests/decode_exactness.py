"""Inputs whose decode attention shows how exactly the probabilities enter, on CPU tensors.

Three tokens a sequence and one element of the queries and keys a head, so that the logits are the numbers
chosen: 0 and two multiples of 1/64 in [-1, 0). The values of a head are bf16 numbers that cancel under the
probabilities to about 2^-16 of their size, so a probability's own error is all that can be seen of the result."""
import torch

TOKENS = 3


def cancelling(seed, R, H, Dh):
    """q [R][H][Dh], k and v [R][H][TOKENS][Dh] in bf16 (a KV head a query head), for a scale of 1."""
    gg = torch.Generator().manual_seed(seed)
    c = torch.cat([torch.zeros(R, H, 1), torch.randint(-64, 0, (R, H, 2), generator=gg) / 64.0], 2).double()
    c = c.gather(2, torch.rand((R, H, TOKENS), generator=gg).argsort(2))
    q, k = torch.zeros(R, H, Dh), torch.zeros(R, H, TOKENS, Dh)
    at = torch.randint(0, Dh, (R, H), generator=gg)
    q.scatter_(2, at[..., None], 1.0)
    k.scatter_(3, at[..., None, None].expand(R, H, TOKENS, 1), c.float()[..., None])
    p = c.exp()[..., None]
    rounded = lambda x: x.to(torch.bfloat16).double()
    v = torch.empty(R, H, TOKENS, Dh, dtype=torch.float64)
    v[:, :, 0] = rounded(1 + torch.rand((R, H, Dh), generator=gg))
    v[:, :, 1] = rounded(-(v[:, :, 0] * p[:, :, 0]) / p[:, :, 1])
    v[:, :, 2] = rounded(-(v[:, :, 0] * p[:, :, 0] + v[:, :, 1] * p[:, :, 1]) / p[:, :, 2])
    return q.bfloat16(), k.bfloat16(), v.bfloat16()


def logits(q, k):
    return (q.double()[:, :, None] * k.double()).sum(-1)


def exact(q, k, v):
    """The output [R][H][Dh] in 64 bits, and its bound.

    With u = 2^-24 and T = sum_j p_j |v_j| / sum_j p_j: a base-2 logit is the product of |s| <= 1 with log2 e,
    that constant and the product rounded (2 u log2 e, as the logit's error a relative 2 u of the
    probability; the largest logit is 0, so nothing is rounded in the difference); the exponential is
    within a step, 2 u. The products of a probability's parts with a value are exact. The leading
    parts' sum takes two additions that round, within a step each if they truncate: 4 u T. It is under 2^-7 T, since
    the leading parts hold 7 bits at least, and so is everything added to it later: 9 more additions are under u T / 8.
    The sum of the probabilities and the division are relative errors of the small result, under 8 u |out|. So 8 u T
    and u T / 8 and half a step of bf16; 9 u T covers them."""
    p = logits(q, k).exp()
    p = (p / p.sum(-1, keepdim=True))[..., None]
    out = (p * v.double()).sum(2)
    return out, 9 * 2.0 ** -24 * (p * v.double().abs()).sum(2) + (2.0 ** -8 + 8 * 2.0 ** -24) * out.abs()


def with_parts(q, k, v, parts):
    """The output where each probability enters as the sum of `parts` bf16 numbers, everything else in 64 bits."""
    p = logits(q, k).exp()
    kept, rest = torch.zeros_like(p), p.clone()
    for _ in range(parts):
        kept += rest.bfloat16().double()
        rest = p - kept
    return ((kept[..., None] * v.double()).sum(2) / p.sum(-1)[..., None]).bfloat16().double()


def repeated(seed, H, Dh, times, dtype):
    """q [1][H][Dh], k and v [1][H][4 times][Dh]: three cancelling tokens and one whose values are 0, over and over.
    Four tokens are a part of every tile, so what is left to cancel outside a tile is a rounding's size."""
    q, k, v = cancelling(seed, 1, H, Dh)
    zero = torch.zeros(1, H, 1, Dh)
    return q.to(dtype), torch.cat([k.float(), zero], 2).repeat(1, 1, times, 1).to(dtype), torch.cat([v.float(), zero], 2).repeat(1, 1, times, 1).to(dtype)


def exact_repeated(q, k, v):
    """As `exact`: 4 u T of the probabilities. A tile of n_t keys is added in n_t (fp32) or 3 n_t (bf16, three parts
    a probability) operations, within a step (2 u) each of what one tile can sum to, its share of T, and the
    tiles' shares add up to T: 2 u n_t T with n_t = 16, 2 u 96 T with 32. Joining waves and parts adds up residues:
    under 2 u T, as does each rescaling's rounding, of which there is none after the largest logit, in the first tile."""
    p = logits(q, k).exp()
    p = (p / p.sum(-1, keepdim=True))[..., None]
    out, T = (p * v.double()).sum(2), (p * v.double().abs()).sum(2)
    u, half, ops = (2.0 ** -24, 2.0 ** -8, 96) if q.dtype == torch.bfloat16 else (2.0 ** -24, 2.0 ** -24, 16)
    return out, (4 + 2 * ops + 4) * u * T + (half + 16 * u) * out.abs()
