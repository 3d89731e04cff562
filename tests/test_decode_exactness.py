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
