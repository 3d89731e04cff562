"""Rows that the rotation and the cache only pass on keep every bit, also those of NaN, infinities and numbers
too small to be normal (needs an MI355X)."""
import numpy as np
import pytest
import torch

from paper_2607_27952_amd import last

pytestmark = pytest.mark.gpu

H, Dh, T, PS = 16, 128, 32, 8


def patterns(dtype):
    """[1][T][H][Dh]: each of the 65536 bf16 numbers once, or 65536 fp32 patterns of every exponent, with the same leading bits."""
    hi = torch.randperm(65536, generator=torch.Generator().manual_seed(7)).to(torch.int32)
    if dtype == torch.bfloat16:
        return hi.to(torch.int16).view(dtype).reshape(1, T, H, Dh)
    lo = torch.randint(0, 65536, (65536,), generator=torch.Generator().manual_seed(8), dtype=torch.int32)
    return ((hi << 16) | lo).view(dtype).reshape(1, T, H, Dh)


def bits(x):
    return x.cpu().contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("turned", [False, True])
def test_append_keeps_bits(dtype, turned):
    """Values always, keys where nothing is turned."""
    x = patterns(dtype)
    cache = last.Cache.make(1, T // PS, PS, H, Dh, dtype)
    pages = last.Pages.make([[2, 0, 3, 1]], [T])
    rot = last.Rotary.make(np.ones(64, np.float32)) if turned else None
    pos = torch.zeros(T, dtype=torch.int32, device="cuda") if turned else None
    k = torch.zeros_like(x) if turned else x
    last.rotary_append(rot, cache, pages, pos, None, k.cuda(), x.cuda(), cu_new_h=[0, T])
    for got, want in ((cache.v, x),) + (() if turned else ((cache.k, x),)):
        rows = got[0, [2, 0, 3, 1]].transpose(1, 2).reshape(1, T, H, Dh)
        assert torch.equal(bits(rows), bits(want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("F", [8, 32, 48])
def test_rotary_keeps_what_it_does_not_turn(dtype, adjacent, F):
    x = patterns(dtype)
    rot = last.Rotary.make(np.ones(F, np.float32), adjacent=adjacent)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    y, z = last.rotary(rot, pos, x.cuda(), x.cuda())
    for got in (y, z):
        assert torch.equal(bits(got[..., 2 * F:]), bits(x[..., 2 * F:]))
