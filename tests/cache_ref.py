"""Plain 64-bit forms of the paged cache's calls, on CPU tensors, and the inputs their tests share."""
import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


def pool(gen, G, pages, Hkv, ps, Dh, dtype, token_major=False):
    """A random pool as [G][pages][Hkv][page][Dh] on the CPU, tokens outermost in a page if asked."""
    if token_major:
        return torch.randn((G, pages, ps, Hkv, Dh), generator=gen).to(dtype).transpose(2, 3)
    return torch.randn((G, pages, Hkv, ps, Dh), generator=gen).to(dtype)


def table_for(rng, lens, ps, spare=2, max_pages=None):
    """Random distinct pages for sequences of these lengths; entries behind the last page name no page.
    Returns the table and how many pages the pool needs (`spare` of them unused)."""
    need = [-(-int(n) // ps) for n in lens]
    ids = rng.permutation(sum(need) + spare).astype(np.int32)
    t = np.full((len(lens), max_pages or max(1, max(need))), 2 ** 30, np.int32)
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = ids[at:at + n]
        at += n
    return t, sum(need) + spare


def rows_of(x, table_row, n):
    """Tokens 0 .. n-1 of a sequence from one layer x [pages][Hkv][page][Dh], as [Hkv][n][Dh] in 64 bits."""
    ps = x.shape[2]
    ids = torch.from_numpy(np.asarray(table_row[:-(-n // ps)], np.int64))
    return x[ids].transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n].double()


def rotary(x, pos, inv_freq, axis, adjacent=False, inverse=False):
    """x [G][T][H][Dh] turned, in 64 bits."""
    F = len(inv_freq)
    a = pos[np.asarray(axis)].double().t() * torch.as_tensor(inv_freq, dtype=torch.float32).double()
    c, s = a.cos()[None, :, None], a.sin()[None, :, None]
    s = -s if inverse else s
    y = x.double().clone()
    if adjacent:
        u, w = y[..., 0:2 * F:2].clone(), y[..., 1:2 * F:2].clone()
        y[..., 0:2 * F:2], y[..., 1:2 * F:2] = u * c - w * s, w * c + u * s
    else:
        u, w = y[..., :F].clone(), y[..., F:2 * F].clone()
        y[..., :F], y[..., F:2 * F] = u * c - w * s, w * c + u * s
    return y


def rotary_bound(x, y, F, adjacent=False):
    """Element-wise bound of a turned row: the angle's reduction in 64 bits (2^31 positions: under 2^-21 of
    a radian), its remainder's rounding and sine and cosine to 4 fp32 steps (2^-22), three fp32 roundings of
    the products and sum (3 * 2^-24), each times |x| + |y| of the pair: 2^-20 in all; and half a step of the output."""
    a = x.double().abs()
    pair = a.clone()
    if adjacent:
        both = a[..., 0:2 * F:2] + a[..., 1:2 * F:2]
        pair[..., 0:2 * F:2], pair[..., 1:2 * F:2] = both, both
    else:
        both = a[..., :F] + a[..., F:2 * F]
        pair[..., :F], pair[..., F:2 * F] = both, both
    pair[..., 2 * F:] = 0
    return pair * 2.0 ** -20 + U[x.dtype] * y.abs() + 2.0 ** -133


def decode(q, k, v, table, lens, scale=0.0):
    """out and lse in 64 bits and their bounds. q [R][Hq][Dh]; k, v one layer [pages][Hkv][page][Dh].

    Per head, with A = max_j sigma sum_d |q_d k_jd| and V = max_j |v_j|: the fp32 logits are within
    (Dh + 8) 2^-23 A (the product's Dh additions at up to a whole step each, the scale, the difference to the
    maximum, the exponential's argument), so weights and their sum are within e = twice that + 2^-22 relative,
    the weights in two bf16 parts within another 2^-16, and n additions at up to a whole step 2^-23 of the sum."""
    R, Hq, Dh = q.shape
    g = Hq // k.shape[1]
    sigma = scale if scale > 0 else 1 / math.sqrt(Dh)
    out, bound = torch.zeros((R, Hq, Dh), dtype=torch.float64), torch.zeros((R, Hq, Dh), dtype=torch.float64)
    lse, lbound = torch.full((R, Hq), -math.inf, dtype=torch.float64), torch.zeros((R, Hq), dtype=torch.float64)
    for r in range(R):
        n = int(lens[r])
        if n == 0:
            continue
        kk = rows_of(k, table[r], n).repeat_interleave(g, 0)
        vv = rows_of(v, table[r], n).repeat_interleave(g, 0)
        qq = q[r].double()
        s = torch.einsum("hd,hnd->hn", qq, kk) * sigma
        lse[r] = torch.logsumexp(s, -1)
        out[r] = torch.einsum("hn,hnd->hd", (s - lse[r][:, None]).exp(), vv)
        A = torch.einsum("hd,hnd->hn", qq.abs(), kk.abs()).amax(-1) * sigma
        e = (Dh + 8) * 2.0 ** -23 * A
        V = vv.abs().amax(1)
        bound[r] = (2 * e + 2.0 ** -22 + 2.0 ** -16 + 2 * n * 2.0 ** -23)[:, None] * V + U[q.dtype] * out[r].abs()
        lbound[r] = e + n * 2.0 ** -23 + 2.0 ** -21 * (1 + lse[r].abs())
    return out, lse, bound, lbound


def prune_index(n_old, vis, N, kept):
    """Old position of every new token; -1 for a kept index outside [0, N)."""
    kept = np.asarray(kept, np.int64)
    mid = np.where((kept >= 0) & (kept < N), vis + kept, -1)
    return np.concatenate([np.arange(vis), mid, np.arange(vis + N, n_old)]).astype(np.int64)


def prune(x, src, dst, ps, old_index):
    """The pool x [G][pages][Hkv][page][Dh] after its sequences were moved; old_index one array per sequence."""
    y = x.clone()
    for r, old in enumerate(old_index):
        for i, o in enumerate(old):
            y[:, dst[r, i // ps], :, i % ps] = x[:, src[r, o // ps], :, o % ps] if o >= 0 else 0
    return y
