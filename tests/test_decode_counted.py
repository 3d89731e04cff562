"""Every cached row counted once: decode attention on inputs that are exact in fp32, at lengths where a bound on
rounding would hide a lost tile. The bound is held to that on the CPU; the rest needs an MI355X."""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
import decode_counted as dc
from paper_2607_27952_amd import last

BF, F32 = torch.bfloat16, torch.float32


def off(got, got_lse, exp):
    """Whether an output or a log-sum-exp lies outside its bound."""
    out, lse, bound, lbound = exp
    return bool(((got - out).abs() > bound).any()) or bool(((got_lse - lse).abs() > lbound).any())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,Hq,Hkv", [(500, 4, 1), (9000, 8, 2), (20001, 7, 1), (36000, 2, 2)])
def test_the_bound_sees_single_rows(dtype, n, Hq, Hkv):
    """Left out, taken twice or weighed with another row's key: every sampled row, tile and page is seen, also
    where the keys or the values alone are wrong."""
    gg, rng = torch.Generator().manual_seed(n), np.random.default_rng(n)
    Dh, ps = 128, 8
    pages = -(-n // ps)
    k, v = dc.pools(gg, 1, pages, Hkv, ps, Dh, dtype)
    q = dc.queries(gg, 1, Hq, Dh, dtype)
    table = rng.permutation(pages).astype(np.int32)[None]
    out, lse, bound, lbound = dc.decode(q, k[0], v[0], table, (n,))
    exp = out[0], lse[0], bound[0], lbound[0]
    kk, vv = ref.rows_of(k[0], table[0], n), ref.rows_of(v[0], table[0], n)
    rounded = lambda x: x.to(dtype).double()
    call = lambda a, b: (lambda o, t: (rounded(o), t.log()))(*dc.attend(q[0].double(), a, b))
    assert not off(*call(kk, vv), exp)
    for at in rng.integers(0, n - 256, 12):
        rows = torch.arange(n)
        one = torch.cat([rows[:at], rows[at + 1:]])
        assert off(*call(kk[:, one], vv[:, one]), exp), "a row left out"
        assert off(*call(torch.cat([kk, kk[:, at:at + 1]], 1), torch.cat([vv, vv[:, at:at + 1]], 1)), exp), "a row twice"
        for tile in (32, 128):
            a = at // tile * tile
            w = vv.clone()
            w[:, a:a + tile] = 0
            assert off(*call(kk, w), exp), "a tile's values missed"
            swapped = rows.clone()
            swapped[a:a + tile], swapped[a + tile:a + 2 * tile] = rows[a + tile:a + 2 * tile], rows[a:a + tile].clone()
            assert off(*call(kk[:, swapped], vv), exp), "two tiles' keys exchanged"
        page = rows.clone()
        a, b = at // ps * ps, (at // ps + 5) * ps
        page[a:a + ps] = rows[b:b + ps]
        assert off(*call(kk, vv[:, page]), exp), "the values of another page"
        assert off(*call(kk[:, page], vv), exp), "the keys of another page"


def up(x):
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x)


def check(cache, pages, q, exp, lens):
    got, lse = last.decode_attention(cache, pages, q.cuda(), scale=dc.SCALE, want_lse=True)
    got, lse = got.cpu().double(), lse.cpu().double()
    assert bool(((got - exp[0]).abs() <= exp[2]).all()), f"out: {int(((got - exp[0]).abs() > exp[2]).sum())} of {got.numel()} off"
    some = torch.from_numpy(np.asarray(lens) > 0)
    assert bool(((lse - exp[1]).abs()[some] <= exp[3][some]).all()), f"lse: worst {float((lse - exp[1]).abs()[some].max()):.3g}"
    assert bool((got[~some] == 0).all()) and bool((lse[~some] == -math.inf).all())


def case(seed, dtype, Dh, Hq, Hkv, ps, lens, major):
    """Pages of NaN behind the sequences' ends and where no sequence lies."""
    gg, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    table, pages = ref.table_for(rng, lens, ps)
    k, v = dc.pools(gg, 1, pages, Hkv, ps, Dh, dtype, major)
    used = torch.zeros((pages, ps), dtype=torch.bool)
    for r, n in enumerate(lens):
        t = np.arange(n)
        used[table[r, t // ps], t % ps] = True
    for p in (k, v):
        p[0].transpose(1, 2)[~used] = math.nan
    q = dc.queries(gg, len(lens), Hq, Dh, dtype)
    return last.Cache(up(k), up(v)), last.Pages.make(table, lens), q, dc.decode(q, k[0], v[0], table, lens)


SHAPES = [(BF, 128, 28, 4, 16, False), (BF, 64, 12, 2, 8, True), (F32, 64, 16, 16, 16, False), (F32, 128, 6, 2, 32, True),
          (BF, 128, 8, 8, 64, True), (BF, 128, 40, 1, 128, False), (BF, 64, 17, 1, 1024, False), (F32, 64, 33, 1, 8, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps,major", SHAPES)
@pytest.mark.parametrize("lens", [(20001, 5, 0, 8191, 8192, 1), (9000,), (1, 2, 31, 32, 33, 127, 128, 129, 255, 257), (2048,) * 3])
def test_every_row_is_counted_once(dtype, Dh, Hq, Hkv, ps, major, lens):
    cache, pages, q, exp = case(len(lens) + Dh, dtype, Dh, Hq, Hkv, ps, lens, major)
    check(cache, pages, q, exp, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps,major", SHAPES[:6])
@pytest.mark.parametrize("R,longest", [(150, 900), (67, 6000)])
def test_ragged_batches(dtype, Dh, Hq, Hkv, ps, major, R, longest):
    rng = np.random.default_rng(R)
    lens = np.exp(rng.uniform(0, math.log(longest), R)).astype(int)
    lens[rng.random(R) < 0.15] = 0
    lens[R // 2] = longest
    lens = tuple(int(n) for n in lens)
    cache, pages, q, exp = case(R, dtype, Dh, Hq, Hkv, ps, lens, major)
    check(cache, pages, q, exp, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("R,major", [(8, False), (16, True)])
def test_stretches_of_more_pages_than_a_block_holds(R, major):
    """More than 1023 pages of 8 tokens in a block's stretch, whose ids are then loaded in turns; a page outside
    the cache in the last of them spoils its sequence only."""
    n, Hkv, Dh, ps, pages = 36000, 16, 64, 8, 3000
    gg, rng = torch.Generator().manual_seed(R), np.random.default_rng(R)
    k, v = dc.pools(gg, 1, pages, Hkv, ps, Dh, BF, major)
    table = rng.integers(0, pages, (R, n // ps)).astype(np.int32)
    q = dc.queries(gg, R, Hkv, Dh, BF)
    cache, lens = last.Cache(up(k), up(v)), [n] * R
    steps = R * Hkv // (2 if major else 1) * -(-n // (64 if major else 128))
    assert steps // (2 * torch.cuda.get_device_properties(0).multi_processor_count) * (64 if major else 128) > 1023 * ps
    out, lse, bound, lbound = dc.decode(q, k[0], v[0], table, lens)
    check(cache, last.Pages.make(table, lens), q, (out, lse, bound, lbound), lens)
    bad = torch.from_numpy(table).cuda()
    bad[3, n // ps - 2] = pages
    seqs = last.Pages(lens_h=np.asarray(lens), table=bad, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    got = last.decode_attention(cache, seqs, q.cuda(), scale=dc.SCALE).cpu().double()
    rest = np.arange(R) != 3
    assert bool(((got - out).abs() <= bound)[rest].all()) and bool(torch.isnan(got[3]).all())
