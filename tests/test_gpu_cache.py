"""Rotary positions, the paged cache and decode attention on the HIP path vs plain
64-bit forms (needs an MI355X). The bounds are derived in cache_ref.py."""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2607_27952_amd import last

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def freqs(F, base=10000.0):
    return (base ** (-np.arange(F) / F)).astype(np.float32)


def up(x):
    """To the GPU with its strides."""
    y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
    y.copy_(x)
    return y


def same_bits(a, b):
    kind = torch.int16 if a.dtype == BF else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def within(got, exp, bound, what=""):
    got = got.detach().cpu().double()
    bad = ~((got - exp).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((got - exp).abs().sub(bound).max()):.3g} over"


# ------------------------------------------------------------------ rotary
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Dh,F,axes,adjacent", [(128, 64, 3, False), (128, 64, 1, True), (64, 32, 3, False),
                                                (64, 16, 2, True), (128, 8, 4, False), (64, 24, 1, False)])
@pytest.mark.parametrize("G,T,Hq,Hkv", [(1, 1, 12, 2), (2, 37, 28, 4), (1, 5, 3, 0), (1, 6, 0, 3), (1, 4097, 2, 1)])
def test_rotary(dtype, Dh, F, axes, adjacent, G, T, Hq, Hkv):
    gg = gen(T + F)
    axis = np.arange(F) % axes
    pos = torch.randint(-2000, 200000, (axes, T), generator=gg, dtype=torch.int32)
    pos[:, 0] = 2 ** 31 - 1
    pos[0, T // 2] = -2 ** 31
    rot = last.Rotary.make(freqs(F), axis=axis, adjacent=adjacent)
    assert rot.n_axes == axes
    q = torch.randn((G, T, Hq, Dh), generator=gg).to(dtype) if Hq else None
    k = torch.randn((G, T, Hkv, Dh), generator=gg).to(dtype) if Hkv else None
    for inverse in (False, True):
        got = last.rotary(rot, pos.cuda(), q.cuda() if Hq else None, k.cuda() if Hkv else None, inverse=inverse)
        for x, y in zip((q, k), got):
            if x is None:
                assert y is None
                continue
            e = ref.rotary(x, pos, freqs(F), axis, adjacent, inverse)
            within(y, e, ref.rotary_bound(x, e, F, adjacent), f"inverse {inverse}")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rotary_of_a_projection_in_place_and_repeated_rows(dtype):
    """q and k as parts of one buffer, turned in place with the values beside them untouched; a broadcast input."""
    G, T, Hq, Hkv, Dh, F = 2, 19, 7, 1, 128, 64
    gg = gen(3)
    qkv = torch.randn((G, T, (Hq + 2 * Hkv) * Dh), generator=gg).to(dtype)
    pos = torch.arange(T, dtype=torch.int32)[None] * 7
    rot = last.Rotary.make(freqs(F))
    d = qkv.cuda()
    q = d[..., :Hq * Dh].unflatten(-1, (Hq, Dh))
    k = d[..., Hq * Dh:(Hq + Hkv) * Dh].unflatten(-1, (Hkv, Dh))
    last.rotary(rot, pos.cuda(), q, k, q_out=q, k_out=k)
    x = qkv[..., :(Hq + Hkv) * Dh].unflatten(-1, (Hq + Hkv, Dh))
    e = ref.rotary(x, pos, freqs(F), np.zeros(F, int))
    within(torch.cat([q, k], 2), e, ref.rotary_bound(x, e, F))
    assert same_bits(d[..., (Hq + Hkv) * Dh:].cpu(), qkv[..., (Hq + Hkv) * Dh:])
    one = torch.randn((1, 1, Hq, Dh), generator=gg).to(dtype)
    many = one.cuda().expand(G, T, Hq, Dh)
    y, _ = last.rotary(rot, pos.cuda(), many)
    e = ref.rotary(one.expand(G, T, Hq, Dh), pos, freqs(F), np.zeros(F, int))
    within(y, e, ref.rotary_bound(one.expand(G, T, Hq, Dh), e, F))


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_inverse_is_the_gradient(adjacent):
    """Against the derivative that 64-bit differentiation of the plain form gives, and against differences of
    the kernel's own forward: for the linear map R, <dy, R(x + h) - R(x)> = <R^T dy, h>."""
    T, H, Dh, F = 9, 4, 64, 24
    gg = gen(5)
    x, dy = torch.randn((1, T, H, Dh), generator=gg), torch.randn((1, T, H, Dh), generator=gg)
    h = torch.randn((1, T, H, Dh), generator=gg)
    pos = torch.randint(0, 5000, (3, T), generator=gg, dtype=torch.int32)
    axis = np.repeat([0, 1, 2], 8)
    rot = last.Rotary.make(freqs(F), sections=(8, 8, 8), adjacent=adjacent)
    leaf = x.double().requires_grad_()
    a = pos[axis].double().t() * torch.from_numpy(freqs(F)).double()
    c, s = a.cos()[None, :, None], a.sin()[None, :, None]
    first, second = (slice(0, 2 * F, 2), slice(1, 2 * F, 2)) if adjacent else (slice(0, F), slice(F, 2 * F))
    u, w = leaf[..., first], leaf[..., second]
    loss = ((u * c - w * s) * dy[..., first].double()).sum() + ((w * c + u * s) * dy[..., second].double()).sum()
    loss = loss + (leaf[..., 2 * F:] * dy[..., 2 * F:].double()).sum()
    loss.backward()
    grad, _ = last.rotary(rot, pos.cuda(), dy.cuda(), inverse=True)
    within(grad, leaf.grad, ref.rotary_bound(dy, leaf.grad, F, adjacent))
    y0, _ = last.rotary(rot, pos.cuda(), x.cuda())
    y1, _ = last.rotary(rot, pos.cuda(), (x + h).cuda())
    left = float((dy.double() * (y1 - y0).cpu().double()).sum())
    right = float((grad.cpu().double() * h.double()).sum())
    # each of the elements of y1, y0 and grad is off by 2^-20 of its pair at most, x + h by 2^-24
    size = float((dy.abs() * 2 * (x.abs() + (x + h).abs() + h.abs()).amax()).double().sum())
    assert abs(left - right) <= 2.0 ** -19 * size


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps,major,adjacent", [
    (BF, 128, 28, 4, 16, False, False), (BF, 64, 12, 2, 8, True, False), (F32, 64, 16, 16, 32, False, True),
    (F32, 128, 3, 1, 64, True, False), (BF, 128, 0, 8, 1024, False, True)])
@pytest.mark.parametrize("new,past", [((1, 1, 1), (0, 15, 16)), ((5, 0, 33), (3, 9, 0)), ((70,), (1,)),
                                      ((1, 1, 1, 1), (7, -1, 3000, 8))])
def test_append(dtype, Dh, Hq, Hkv, ps, major, adjacent, new, past):
    """Every place of both pools: new rows at their tokens, the rest untouched; an empty slot (past -1, so
    that its length is 0) stores nothing."""
    gg, rng = gen(len(new) + ps), np.random.default_rng(ps)
    G, layer, n_layers, F = 2, 1, 4, Dh // 4
    lens = np.asarray([a + b for a, b in zip(new, past)], np.int32)
    T = sum(new)
    table, pages = ref.table_for(rng, lens, ps)
    kp, vp = (ref.pool(gg, n_layers, pages, Hkv, ps, Dh, dtype, major) for _ in "kv")
    cache = last.Cache(up(kp), up(vp))
    pos = torch.randint(0, 40000, (3, T), generator=gg, dtype=torch.int32)
    axis = np.repeat([0, 1, 2], [F // 4, F // 4, F - 2 * (F // 4)])
    rot = last.Rotary.make(freqs(F), axis=axis, adjacent=adjacent)
    q = torch.randn((G, T, Hq, Dh), generator=gg).to(dtype) if Hq else None
    k, v = (torch.randn((G, T, Hkv, Dh), generator=gg).to(dtype) for _ in "kv")
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    kw = {} if all(n == 1 for n in new) and past[0] == 0 else {"cu_new_h": cu}
    q_out = last.rotary_append(rot, cache, last.Pages.make(table, lens), pos.cuda(), q.cuda() if Hq else None, k.cuda(),
                               v.cuda(), layer=layer, **kw)
    if Hq:
        e = ref.rotary(q, pos, freqs(F), axis, adjacent)
        within(q_out, e, ref.rotary_bound(q, e, F, adjacent))
    e = ref.rotary(k, pos, freqs(F), axis, adjacent)
    exp_k, exp_v, tol = kp.double(), vp.clone(), torch.zeros(kp.shape, dtype=torch.float64)
    b = ref.rotary_bound(k, e, F, adjacent)
    for r, n in enumerate(new):
        for i in range(n):
            at, t = past[r] + i, cu[r] + i
            if at < 0:
                continue
            page = table[r, at // ps]
            exp_k[layer:layer + G, page, :, at % ps] = e[:, t]
            tol[layer:layer + G, page, :, at % ps] = b[:, t]
            exp_v[layer:layer + G, page, :, at % ps] = v[:, t]
    within(cache.k, exp_k, tol, "keys")
    assert same_bits(cache.v.cpu(), exp_v)


def test_append_without_rotation_and_past_the_bound():
    """rot None stores keys bit for bit; a length behind the bound, or a page outside the cache, stores nothing."""
    gg = gen(8)
    R, Hkv, Dh, ps = 4, 2, 64, 8
    kp, vp = (ref.pool(gg, 1, 6, Hkv, ps, Dh, BF) for _ in "kv")
    cache = last.Cache(kp.cuda(), vp.cuda())
    table = np.asarray([[0, 1], [2, 3], [4, 9], [5, 5]], np.int32)
    lens = np.asarray([9, 17, 9, 1], np.int32)       # 17 is behind the bound 16, table[2][1] names no page
    pages = last.Pages(lens_h=np.asarray([16, 16, 16, 16]), table=torch.from_numpy(table).cuda(),
                       lens=torch.from_numpy(lens).cuda())
    k, v = (torch.randn((1, R, Hkv, Dh), generator=gg).to(BF) for _ in "kv")
    assert last.rotary_append(None, cache, pages, None, None, k.cuda(), v.cuda()) is None
    for x, p, got in ((k, kp, cache.k), (v, vp, cache.v)):
        p[0, 1, :, 0] = x[0, 0]
        p[0, 5, :, 0] = x[0, 3]
        assert same_bits(got.cpu(), p)


# ------------------------------------------------------------------ decode
def decode_case(seed, dtype, Dh, Hq, Hkv, ps, lens, major=False, spread=1.0, G=2, layer=1, scale=0.0, bound=None):
    gg, rng = gen(seed), np.random.default_rng(seed)
    table, pages = ref.table_for(rng, lens, ps)
    kp, vp = (ref.pool(gg, G, pages, Hkv, ps, Dh, dtype, major) for _ in "kv")
    q = (torch.randn((len(lens), Hq, Dh), generator=gg) * spread).to(dtype)
    exp = ref.decode(q, kp[layer], vp[layer], table, lens, scale)
    # nothing behind a sequence's end, in another layer or in an unused page may matter
    used = torch.zeros((pages, ps), dtype=torch.bool)
    for r, n in enumerate(lens):
        for t in range(n):
            used[table[r, t // ps], t % ps] = True
    for p in (kp, vp):
        p[:layer] = math.nan
        p[layer].transpose(1, 2)[~used] = math.nan
    cache = last.Cache(up(kp), up(vp))
    if bound is None:
        pages = last.Pages.make(table, lens)
    else:
        pages = last.Pages(lens_h=np.minimum(bound, table.shape[1] * ps), table=torch.from_numpy(table).cuda(),
                           lens=torch.tensor(lens, dtype=torch.int32).cuda())
    return cache, pages, q, exp


SHAPES = [(BF, 128, 28, 4, 16, False), (BF, 64, 12, 2, 8, True), (F32, 64, 16, 16, 16, False), (F32, 128, 6, 2, 32, True),
          (BF, 128, 32, 32, 64, True), (BF, 128, 17, 1, 128, False), (BF, 64, 40, 1, 1024, False),
          (F32, 128, 33, 1, 8, False)]


@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps,major", SHAPES)
@pytest.mark.parametrize("lens", [(1,), (0, 3, 0), (31, 32, 33, 127, 128, 129), (1000, 1, 513, 0), (2500,)])
def test_decode(dtype, Dh, Hq, Hkv, ps, major, lens):
    cache, pages, q, (out, lse, ob, lb) = decode_case(sum(lens) + Dh, dtype, Dh, Hq, Hkv, ps, lens, major)
    got, got_lse = last.decode_attention(cache, pages, q.cuda(), layer=1, want_lse=True)
    within(got, out, ob, "out")
    for r, n in enumerate(lens):
        if n == 0:
            assert bool((got[r] == 0).all()) and bool((got_lse[r] == -math.inf).all())
    some = np.asarray(lens) > 0
    within(got_lse[some], lse[some], lb[some], "lse")
    again = last.decode_attention(cache, pages, q.cuda(), layer=1)
    assert same_bits(again.cpu(), got.cpu()), "two runs differ"


@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps", [(BF, 128, 28, 4, 16), (BF, 64, 8, 8, 256), (F32, 128, 8, 2, 8)])
def test_decode_long_ragged(dtype, Dh, Hq, Hkv, ps):
    lens = (20001, 5, 0, 8191, 8192, 1)
    cache, pages, q, (out, lse, ob, lb) = decode_case(77, dtype, Dh, Hq, Hkv, ps, lens, G=1, layer=0)
    got, got_lse = last.decode_attention(cache, pages, q.cuda(), want_lse=True)
    within(got, out, ob, "out")
    some = np.asarray(lens) > 0
    within(got_lse[some], lse[some], lb[some], "lse")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("spread,scale", [(40.0, 0.0), (0.0, 0.0), (1.0, 3.0)])
def test_decode_sharp_flat_and_scaled(dtype, spread, scale):
    """Logits of hundreds, all equal, and another scale."""
    lens = (600, 3, 4000)
    cache, pages, q, (out, lse, ob, lb) = decode_case(5, dtype, 128, 8, 2, 16, lens, spread=spread, scale=scale)
    got, got_lse = last.decode_attention(cache, pages, q.cuda(), layer=1, scale=scale, want_lse=True)
    within(got, out, ob, "out")
    within(got_lse, lse, lb, "lse")


@pytest.mark.parametrize("n", [40, 3000])
def test_decode_minus_infinity(n):
    """Keys whose logit is -inf get no weight, also where whole tiles hold nothing else; NaN in one key's
    logit spoils its sequence only."""
    Dh, ps = 128, 16
    rng, gg = np.random.default_rng(1), gen(1)
    table, pages = ref.table_for(rng, (n, n, n), ps)
    kp, vp = (ref.pool(gg, 1, pages, 1, ps, Dh, BF) for _ in "kv")
    q = torch.randn((3, 4, Dh), generator=gg).to(BF)
    q[..., 0] = 1.0
    keep = np.zeros(n, bool)
    keep[[n - 1, n // 2]] = True
    kp[0, :, 0, :, 0] = 0.0
    for t in range(n):
        if not keep[t]:
            kp[0, table[0, t // ps], 0, t % ps, 0] = -math.inf
    kp[0, table[2, 0], 0, 3, 5] = math.nan
    got = last.decode_attention(last.Cache(kp.cuda(), vp.cuda()), last.Pages.make(table, (n, n, n)), q.cuda()).cpu()
    k = ref.rows_of(kp[0], table[0], n)[0][keep]
    v = ref.rows_of(vp[0], table[0], n)[0][keep]
    w = torch.softmax(q[0].double() @ k.t() / math.sqrt(Dh), -1)
    # as in cache_ref.decode with A under 40: (Dh + 8) 2^-22 A, 2^-16, and half a step
    exp = w @ v
    within(got[0], exp, ((Dh + 8) * 2.0 ** -22 * 40 + 2.0 ** -15 + n * 2.0 ** -22) * v.abs().amax() + 2.0 ** -8 * exp.abs())
    out, _, ob, _ = ref.decode(q[1:2], kp[0], vp[0], table[1:2], (n,))
    within(got[1:2], out, ob)
    assert bool(torch.isnan(got[2]).all())


@pytest.mark.parametrize("n", [100, 5000])
def test_decode_bad_page_is_not_followed(n):
    """A page outside the cache, met only by the kernel's own check (no host table): its sequence gives NaN,
    the others what they gave."""
    cache, pages, q, (out, lse, ob, lb) = decode_case(9, BF, 64, 4, 2, 16, (n, n, n), G=1, layer=0)
    table = pages.table.clone()
    table[1, (n - 1) // 16] = cache.k.shape[1]
    table[2, 0] = -1
    broken = last.Pages(lens_h=pages.lens_h, table=table, lens=pages.lens)
    got, got_lse = last.decode_attention(cache, broken, q.cuda(), want_lse=True)
    within(got[:1], out[:1], ob[:1])
    assert bool(torch.isnan(got[1:]).all()) and bool(torch.isnan(got_lse[1:]).all())
    assert not bool(torch.isnan(got_lse[0]).any())


def test_decode_bounds_and_buffers():
    """Lengths below their bounds, a bound exceeded (cut to it), q as part of a wider buffer, and out with rows
    behind the last sequence."""
    lens = (700, 0, 33, 1500)
    cache, pages, q, (out, lse, ob, lb) = decode_case(21, BF, 128, 28, 4, 16, lens, bound=np.asarray([1504, 1504, 40, 1500]))
    wide = torch.full((4, 28 * 128 + 512), math.nan, dtype=BF, device="cuda")
    wide[:, :28 * 128] = q.reshape(4, -1).cuda()
    buf = torch.full((6, 28, 128), 7.0, dtype=BF, device="cuda")
    last.decode_attention(cache, pages, wide[:, :28 * 128].unflatten(1, (28, 128)), layer=1, out=buf[:4])
    within(buf[:4], out, ob)
    assert bool((buf[4:] == 7.0).all())
    over = pages.lens.clone()
    over[0] = 2 ** 31 - 1
    over[2] = -5
    got = last.decode_attention(cache, last.Pages(lens_h=np.asarray([700, 1, 40, 700]), table=pages.table, lens=over),
                                q.cuda(), layer=1)
    within(got[0], out[0], ob[0])      # cut to the largest bound, 700
    assert bool((got[1:3] == 0).all())


def test_decode_far_pages():
    """Pages whose elements lie past 2^31 in the pool."""
    ps, Hkv, Dh = 16, 8, 128
    per = Hkv * ps * Dh
    pages = 2 ** 31 // per + 40
    gg, rng = gen(2), np.random.default_rng(2)
    kd, vd = (torch.empty((1, pages, Hkv, ps, Dh), dtype=BF, device="cuda") for _ in "kv")
    n = 300
    ids = np.asarray([pages - 1 - i for i in rng.permutation(20)] + [0], np.int32)[-19:][None]
    ids = np.ascontiguousarray(ids)
    small_k, small_v = (torch.randn((19, Hkv, ps, Dh), generator=gg).to(BF) for _ in "kv")
    at = torch.from_numpy(ids[0].astype(np.int64)).cuda()
    kd[0, at], vd[0, at] = small_k.cuda(), small_v.cuda()
    q = torch.randn((1, 16, Dh), generator=gg).to(BF)
    cache = last.Cache(kd, vd)
    got = last.decode_attention(cache, last.Pages.make(ids, (n,)), q.cuda())
    out, _, ob, _ = ref.decode(q, small_k, small_v, np.arange(19)[None], (n,))
    within(got, out, ob)
    last.cache_copy(cache, ids[0, :2], [1, 2])
    assert same_bits(kd[0, 1:3].cpu(), small_k[:2]) and same_bits(vd[0, 1:3].cpu(), small_v[:2])


# ------------------------------------------------------------------ pages
@pytest.mark.parametrize("dtype,Dh,Hkv,ps,major,G", [(BF, 128, 4, 16, False, 3), (BF, 64, 3, 8, True, 1), (F32, 64, 1, 32, False, 2),
                                                     (F32, 128, 5, 64, True, 2)])
def test_copy(dtype, Dh, Hkv, ps, major, G):
    gg, rng = gen(4), np.random.default_rng(4)
    kp, vp = (ref.pool(gg, G, 40, Hkv, ps, Dh, dtype, major) for _ in "kv")
    for n in (0, 1, 17):
        ids = rng.permutation(40)
        src, dst = ids[:n], ids[20:20 + n]
        src = np.where(np.arange(n) == n - 1, src[:1], src) if n > 1 else src     # one page copied twice
        cache = last.Cache(up(kp), up(vp))
        last.cache_copy(cache, src, dst)
        for p, got in ((kp, cache.k), (vp, cache.v)):
            e = p.clone()
            e[:, dst] = p[:, src]
            assert same_bits(got.cpu(), e)


def test_copy_of_interleaved_keys_and_values():
    """Keys and values of a token side by side in one buffer, heads padded: both views share their strides."""
    gg = gen(6)
    buf = torch.randn((2, 9, 16, 3, 2, 80), generator=gg).to(BF)     # layer, page, token, head, k or v, Dh + 16
    d = buf.cuda()
    cache = last.Cache(*(d[..., i, :64].transpose(2, 3) for i in (0, 1)))
    last.cache_copy(cache, [0, 3], [8, 5])
    e = buf.clone()
    e[:, [8, 5], ..., :64] = buf[:, [0, 3], ..., :64]
    assert same_bits(d.cpu(), e)


@pytest.mark.parametrize("dtype,Dh,Hkv,ps,major,G", [(BF, 128, 4, 16, False, 2), (BF, 64, 2, 8, True, 1), (F32, 64, 16, 32, False, 2),
                                                     (F32, 128, 3, 64, True, 1)])
@pytest.mark.parametrize("shapes", [
    [(40, 5, 30, 4)], [(100, 0, 90, 90), (20, 3, 10, 0), (50, 20, 0, 0)], [(0, 0, 0, 0), (33, 16, 16, 3), (300, 40, 200, 25)],
    [(16, 0, 16, 1)]])
def test_prune(dtype, Dh, Hkv, ps, major, G, shapes):
    """Sequences of (tokens, start of the visual ones, their number, kept): every place of both pools."""
    gg, rng = gen(len(shapes)), np.random.default_rng(len(shapes))
    lens = [s[0] for s in shapes]
    after = [n - N + K for n, _, N, K in shapes]
    table, _ = ref.table_for(rng, lens + after, ps, max_pages=-(-max(lens + after + [1]) // ps) + 1)
    pages = int(table[table < 2 ** 30].max(initial=0)) + 3
    src, dst = np.ascontiguousarray(table[:len(lens)]), np.ascontiguousarray(table[len(lens):])
    kp, vp = (ref.pool(gg, G, pages, Hkv, ps, Dh, dtype, major) for _ in "kv")
    kept = [np.sort(rng.choice(N, K, replace=False)) for _, _, N, K in shapes]
    vis = [s[1] for s in shapes]
    cu_vis, cu_keep = (np.concatenate([[0], np.cumsum([s[i] for s in shapes])]) for i in (2, 3))
    cache = last.Cache(up(kp), up(vp))
    flat = torch.tensor(np.concatenate(kept), dtype=torch.int32).cuda()
    into = last.Pages.make(dst, after)
    into.lens.fill_(-7)
    got = last.cache_prune(cache, last.Pages.make(src, lens), into, vis, cu_vis, flat, cu_keep)
    assert got is into.lens and got.tolist() == after
    old = [ref.prune_index(s[0], s[1], s[2], k) for s, k in zip(shapes, kept)]
    for p, x in ((kp, cache.k), (vp, cache.v)):
        assert same_bits(x.cpu(), ref.prune(p, src, dst, ps, old))


def test_prune_shares_whole_pages_and_zeroes_bad_indices():
    """Two continuations of one prompt, pruned differently, whose first pages stay shared; an index outside the
    visual tokens gives a row of zeros."""
    gg, ps = gen(12), 8
    kp, vp = (ref.pool(gg, 2, 30, 2, ps, 64, BF) for _ in "kv")
    n, vis, N = 70, 20, 40
    src = np.asarray([[3, 1, 4, 2, 9, 6, 5, 8, 7], [3, 1, 4, 2, 9, 6, 5, 8, 7]], np.int32)
    kept = np.asarray([0, 7, 39, 3, -1, 40], np.int32)
    dst = np.asarray([[3, 1, 20, 21, 22], [3, 1, 23, 24, 25]], np.int32)
    after = [n - N + 3] * 2
    cache = last.Cache(kp.cuda(), vp.cuda())
    last.cache_prune(cache, last.Pages.make(src, [n, n]), last.Pages.make(dst, after), [vis, vis], [0, N, 2 * N],
                     torch.from_numpy(kept).cuda(), [0, 3, 6])
    old = [ref.prune_index(n, vis, N, k) for k in (kept[:3], kept[3:])]
    for p, x in ((kp, cache.k), (vp, cache.v)):
        assert same_bits(x.cpu(), ref.prune(p, src, dst, ps, old))


# ------------------------------------------------------------------ together
def prompt(seed, dtype=BF, G=2, Hq=8, Hkv=2, Dh=128, lens=(90, 150), vis=(10, 20), N=(60, 100), K=(12, 9)):
    gg = gen(seed)
    T = sum(lens)
    raw = {n: torch.randn((G, T, h, Dh), generator=gg).to(dtype) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    pos = torch.stack([torch.cat([torch.arange(n) // d for n in lens]) for d in (1, 4, 7)]).int()
    return raw, pos


def test_prompt_to_answer():
    """The calls as they are used: a prompt's q and k turned and put into the cache, its prefill attention and
    scores, the k-center's choice, the cache pruned to it, then tokens decoded from the pruned cache; every
    step against the 64-bit forms on what the step before it gave."""
    G, Hq, Hkv, Dh, ps = 2, 8, 2, 128, 16
    lens, vis, N, K = (90, 150), (10, 20), (60, 100), (12, 9)
    raw, pos = prompt(31)
    F, axis = 64, np.repeat([0, 1, 2], [16, 24, 24])
    rot = last.Rotary.make(freqs(F), sections=(16, 24, 24))
    cu = np.concatenate([[0], np.cumsum(lens)])
    cu_vis, cu_keep = np.concatenate([[0], np.cumsum(N)]), np.concatenate([[0], np.cumsum(K)])
    rng = np.random.default_rng(31)
    after = [n - a + b for n, a, b in zip(lens, N, K)]
    steps = 20
    table, pages = ref.table_for(rng, list(lens) + [a + steps for a in after], ps, max_pages=10)
    src, dst = np.ascontiguousarray(table[:2]), np.ascontiguousarray(table[2:])
    cache = last.Cache.make(G, pages, ps, Hkv, Dh)
    cache.k.fill_(math.nan), cache.v.fill_(math.nan)
    full = last.Pages.make(src, lens)

    q, k, v = (raw[n].cuda() for n in "qkv")
    q = last.rotary_append(rot, cache, full, pos.cuda(), q, k, v, cu_new_h=cu)
    turned = torch.stack([torch.cat([ref.rows_of(cache.k[g].cpu(), src[r], lens[r]).transpose(0, 1) for r in range(2)])
                          for g in range(G)])
    e = ref.rotary(raw["k"], pos, freqs(F), axis)
    within(turned, e, ref.rotary_bound(raw["k"], e, F), "cached keys")

    batch = last.Batch.make(G, Hq, Hkv, Dh, cu, vis, cu_vis)
    out, scores = last.prefill_attention(batch, q, turned.to(BF).cuda(), v)
    # the prefill's last rows are what decoding the last token over the whole cache gives
    rows = cu[1:] - 1
    for g in range(G):
        got = last.decode_attention(cache, full, q[g, rows].contiguous(), layer=g)
        exp, _, ob, _ = ref.decode(q[g, rows].cpu(), cache.k[g].cpu(), cache.v[g].cpu(), src, lens)
        within(got, exp, ob, "last rows")
        vmax = raw["v"][g].double().abs().amax()
        within(out[g, rows], exp, ob + 2.0 ** -8 * vmax, "prefill")      # its probabilities are rounded to bf16

    feats = torch.randn((sum(N), 256), generator=gen(1)).to(BF).cuda()
    kept, _, _ = last.diverse_select(scores, feats, cu_vis, cu_keep)
    before = cache.k.cpu(), cache.v.cpu()
    pruned = last.Pages(table_h=dst, lens_h=np.asarray([a + steps for a in after]), table=torch.from_numpy(dst).cuda(),
                        lens=torch.zeros(2, dtype=torch.int32, device="cuda"))
    last.cache_prune(cache, full, pruned, vis, cu_vis, kept, cu_keep)
    old = [ref.prune_index(lens[r], vis[r], N[r], kept[cu_keep[r]:cu_keep[r + 1]].cpu().numpy()) for r in range(2)]
    for was, now in zip(before, (cache.k, cache.v)):
        assert same_bits(now.cpu(), ref.prune(was, src, dst, ps, old))

    gg = gen(32)
    for step in range(steps):
        pruned.lens.add_(1)
        now = [a + step + 1 for a in after]
        p = torch.tensor([lens], dtype=torch.int32).expand(3, 2).contiguous() + step
        for g in range(G):
            x = {n: torch.randn((1, 2, h, Dh), generator=gg).to(BF) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
            qt = last.rotary_append(rot, cache, pruned, p.cuda(), x["q"].cuda(), x["k"].cuda(), x["v"].cuda(), layer=g)
            got = last.decode_attention(cache, pruned, qt[0], layer=g)
            if step % 6 == 0 or step == steps - 1:
                e = ref.rotary(x["k"], p, freqs(F), axis)
                b = ref.rotary_bound(x["k"], e, F)
                for r in range(2):
                    at = now[r] - 1
                    within(cache.k[g, dst[r, at // ps], :, at % ps], e[0, r], b[0, r], "new key")
                exp, _, ob, _ = ref.decode(qt[0].cpu(), cache.k[g].cpu(), cache.v[g].cpu(), dst, now)
                within(got, exp, ob, f"step {step}")


class CapturedStep:
    """One decoding step captured over a cache of its own, and the same step run eagerly on a copy of it."""
    R, Hq, Hkv, Dh, ps = 3, 12, 2, 128, 16

    def __init__(self, seed, start, steps):
        self.gen, rng = gen(seed), np.random.default_rng(seed)
        R, Hq, Hkv, Dh, ps = self.R, self.Hq, self.Hkv, self.Dh, self.ps
        bound = np.asarray([start + steps, 5 + steps, start // 2 + steps], np.int32)
        table, pages = ref.table_for(rng, bound, ps)
        self.cache = last.Cache(*(ref.pool(self.gen, 1, pages, Hkv, ps, Dh, BF).cuda() for _ in "kv"))
        self.copy = last.Cache(self.cache.k.clone(), self.cache.v.clone())
        self.rot = last.Rotary.make(freqs(64))
        self.pages = last.Pages(table_h=table, lens_h=bound, table=torch.from_numpy(table).cuda(),
                                lens=torch.from_numpy(bound - steps).cuda())
        self.x = {n: torch.zeros((1, R, h, Dh), dtype=BF, device="cuda") for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
        self.pos = torch.zeros((1, R), dtype=torch.int32, device="cuda")
        self.turned = torch.empty_like(self.x["q"])
        need = last.decode_attention_workspace(self.cache, self.pages, Hq)
        self.ws, self.other_ws = (torch.empty(need, dtype=torch.uint8, device="cuda") for _ in "ab")
        self.out, self.other_out = (torch.empty((R, Hq, Dh), dtype=BF, device="cuda") for _ in "ab")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step(self.copy, self.other_out, self.other_ws)    # the first launch of each kernel, not captured
        torch.cuda.current_stream().wait_stream(side)
        self.pages.lens.sub_(1)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step(self.cache, self.out, self.ws)

    def step(self, cache, out, ws):
        self.pages.lens.add_(1)
        self.pos.copy_(self.pages.lens[None])
        last.rotary_append(self.rot, cache, self.pages, self.pos, self.x["q"], self.x["k"], self.x["v"], q_out=self.turned)
        last.decode_attention(cache, self.pages, self.turned[0], out=out, ws=ws)


@pytest.mark.parametrize("start", [30, 1200])
def test_captured_steps(start):
    """Two captured decoding steps with workspaces of their own, replayed in turn while their lengths grow,
    equal to eager calls bit for bit; other work runs between the replays."""
    steps = 6
    sides = [CapturedStep(seed, start, steps) for seed in (1, 2)]
    for i in range(steps):
        for c in sides:
            for t in c.x.values():
                t.copy_(torch.randn(t.shape, generator=c.gen).to(BF))
            c.graph.replay()
            got = c.out.clone()
            torch.cuda.synchronize()
            c.pages.lens.sub_(1)
            c.step(c.copy, c.other_out, c.other_ws)
            assert same_bits(got.cpu(), c.other_out.cpu()), f"replay {i}"
            assert not bool(torch.isnan(got).any())


def test_calls_on_a_stream_of_their_own():
    """Everything enqueued on a side stream while the current one is busy elsewhere."""
    cache, pages, q, (out, lse, ob, lb) = decode_case(14, BF, 128, 8, 2, 16, (900, 30))
    s = torch.cuda.Stream()
    x = q.cuda()
    torch.cuda.synchronize()
    got = last.decode_attention(cache, pages, x, layer=1, stream=s)
    pos = torch.arange(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    y, _ = last.rotary(last.Rotary.make(freqs(64)), pos, x[None], stream=s)
    s.synchronize()
    within(got, out, ob)
    e = ref.rotary(q[None], pos.cpu()[None], freqs(64), np.zeros(64, int))
    within(y, e, ref.rotary_bound(q[None], e, 64))
