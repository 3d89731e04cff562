"""How exactly the probabilities of the decode attention enter the value product: the bound on the CPU, and the
kernel (needs an MI355X)."""
import numpy as np
import pytest
import torch

import decode_exactness as de
from paper_2607_27952_amd import last


def over(got, exp, bound):
    return int(((got - exp).abs() > bound).sum())


@pytest.mark.parametrize("Dh", [64, 128])
def test_the_bound_sees_sixteen_bits(Dh):
    """Two bf16 numbers a probability are seen, three pass."""
    q, k, v = de.cancelling(3, 64, 8, Dh)
    exp, bound = de.exact(q, k, v)
    assert over(de.with_parts(q, k, v, 1), exp, bound) > 0.5 * exp.numel()
    assert over(de.with_parts(q, k, v, 2), exp, bound) > 0.01 * exp.numel()
    assert over(de.with_parts(q, k, v, 3), exp, bound) == 0
    assert float(exp.abs().max()) < 2.0 ** -13      # the values do cancel


@pytest.mark.gpu
@pytest.mark.parametrize("Dh,ps,major", [(128, 16, False), (64, 8, False), (128, 8, True), (64, 32, True)])
@pytest.mark.parametrize("R", [1, 64, 200])
def test_probabilities_keep_their_bits(Dh, ps, major, R):
    H = 8
    q, k, v = de.cancelling(5 + R, R, H, Dh)
    pools = []
    for x in (k, v):
        pool = torch.full((1, R, ps, H, Dh) if major else (1, R, H, ps, Dh), float("nan"), dtype=torch.bfloat16)
        pool = pool.transpose(2, 3) if major else pool
        pool[0, :, :, :de.TOKENS] = x
        pools.append(torch.empty_strided(pool.shape, pool.stride(), dtype=pool.dtype, device="cuda").copy_(pool))
    pages = last.Pages.make(np.arange(R, dtype=np.int32)[:, None], [de.TOKENS] * R)
    got = last.decode_attention(last.Cache(*pools), pages, q.cuda(), scale=1.0)
    exp, bound = de.exact(q, k, v)
    bad = over(got.cpu().double(), exp, bound)
    assert bad == 0, f"{bad} of {exp.numel()} off, worst {float(((got.cpu().double() - exp).abs() / bound).max()):.3g} bounds"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("times", [1, 150, 2500])
def test_the_bound_sees_eight_bits_at_any_length(dtype, times):
    """A probability rounded to one bf16 number is seen in sequences of 4 to 10000 tokens."""
    q, k, v = de.repeated(9, 8, 128, times, dtype)
    exp, bound = de.exact_repeated(q, k, v)
    assert over(de.with_parts(q, k, v, 1), exp, bound) > 0.5 * exp.numel()
    p = de.logits(q, k).exp()
    whole = ((p[..., None] * v.double()).sum(2) / p.sum(-1)[..., None]).to(dtype).double()
    assert over(whole, exp, bound) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("times", [1, 9, 150, 700, 2500])
@pytest.mark.parametrize("Dh,ps,major", [(128, 16, False), (64, 8, True), (128, 64, True)])
def test_probabilities_keep_their_bits_at_any_length(dtype, times, Dh, ps, major):
    H, n = 8, 4 * times
    q, k, v = de.repeated(9 + times, H, Dh, times, dtype)
    pages = -(-n // ps)
    table = np.random.default_rng(times).permutation(pages).astype(np.int32)
    pools = []
    for x in (k, v):
        flat = torch.full((H, pages * ps, Dh), float("nan"), dtype=dtype)
        flat[:, :n] = x[0]
        flat = flat.view(H, pages, ps, Dh)
        pool = torch.empty((pages, ps, H, Dh) if major else (pages, H, ps, Dh), dtype=dtype, device="cuda")
        (pool.transpose(1, 2) if major else pool)[torch.from_numpy(table.astype(np.int64)).cuda()] = flat.transpose(0, 1).cuda()
        pools.append((pool.transpose(1, 2) if major else pool)[None])
    got = last.decode_attention(last.Cache(*pools), last.Pages.make(table[None], [n]), q.cuda(), scale=1.0).cpu().double()
    exp, bound = de.exact_repeated(q, k, v)
    assert over(got, exp, bound) == 0, f"worst {float(((got - exp).abs() / bound).max()):.3g} bounds"
