"""The cache's calls where they change how they lay their work out (needs an MI355X): batches past a wave of
sequences, blocks that serve several sequences, heads beside each other, several tokens, layers or batches of
rows a block. Bounds as in cache_ref.py."""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2607_27952_amd import last
from test_gpu_cache import BF, F32, decode_case, freqs, gen, same_bits, up, within

pytestmark = pytest.mark.gpu


def check(cache, pages, q, exp, lens, layer):
    out, lse, ob, lb = exp
    got, got_lse = last.decode_attention(cache, pages, q.cuda(), layer=layer, want_lse=True)
    within(got, out, ob, "out")
    some = np.asarray(lens) > 0
    within(got_lse[some], lse[some], lb[some], "lse")
    assert bool((got_lse[~torch.from_numpy(some)] == -math.inf).all()) and bool((got[~torch.from_numpy(some)] == 0).all())
    again, again_lse = last.decode_attention(cache, pages, q.cuda(), layer=layer, want_lse=True)
    assert same_bits(again, got) and same_bits(again_lse, got_lse)


@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps,major", [
    (BF, 128, 4, 2, 16, True), (BF, 128, 3, 3, 32, True), (BF, 64, 36, 2, 8, True), (F32, 64, 8, 8, 16, True),
    (BF, 128, 14, 2, 64, False), (F32, 128, 20, 1, 256, False)])
@pytest.mark.parametrize("R,longest", [(150, 900), (67, 4000), (3, 9000)])
def test_decode_batches(dtype, Dh, Hq, Hkv, ps, major, R, longest):
    """Many sequences of very different lengths, empty ones between them: stretches of the line that end, begin
    and lie inside units, and units of one part, two and many."""
    r = np.random.default_rng(R + Dh)
    lens = np.exp(r.uniform(0, math.log(longest), R)).astype(int)
    lens[r.random(R) < 0.15] = 0
    lens[-1 if R > 100 else 0] = longest
    cache, pages, q, exp = decode_case(R, dtype, Dh, Hq, Hkv, ps, tuple(int(n) for n in lens), major, G=1, layer=0)
    check(cache, pages, q, exp, lens, 0)


@pytest.mark.parametrize("lens", [(0,) * 70, (1,) + (0,) * 69, (0,) * 69 + (200,), (3, 0) * 35])
@pytest.mark.parametrize("major", [False, True])
def test_decode_far_below_the_bounds(lens, major):
    """A call laid out for long sequences whose lengths on the device are short: fewer steps than blocks."""
    R, ps, Hkv, Dh = len(lens), 16, 2, 128
    gg = gen(3)
    table = np.tile(np.arange(128, dtype=np.int32), (R, 1))      # sequences may share pages
    kp, vp = (ref.pool(gg, 1, 128, Hkv, ps, Dh, BF, major) for _ in "kv")
    q = torch.randn((R, 12, Dh), generator=gg).to(BF)
    pages = last.Pages(lens_h=np.asarray([2048] * 20 + [300] * (R - 20)), table=torch.from_numpy(table).cuda(),
                       lens=torch.tensor(lens, dtype=torch.int32).cuda())
    check(last.Cache(up(kp), up(vp)), pages, q, ref.decode(q, kp[0], vp[0], table, lens), lens, 0)


def test_decode_shared_workspace_of_unlike_calls():
    """One workspace for calls of unlike shapes one after the other, full of NaN at first."""
    cases = [decode_case(41, BF, 128, 28, 4, 16, (3000, 40, 0), G=1, layer=0),
             decode_case(42, BF, 64, 12, 2, 8, (1, 1999), True, G=1, layer=0),
             decode_case(43, F32, 128, 6, 2, 32, (777,), True, G=1, layer=0)]
    need = max(last.decode_attention_workspace(c[0], c[1], c[2].shape[1]) for c in cases)
    ws = torch.full((need // 4,), math.nan, device="cuda")
    for cache, pages, q, (out, _, ob, _) in cases + cases[::-1]:
        within(last.decode_attention(cache, pages, q.cuda(), ws=ws), out, ob)


@pytest.mark.parametrize("dtype,Dh,Hq,Hkv,ps,major,adjacent", [(BF, 64, 3, 1, 16, False, False), (F32, 64, 2, 2, 8, True, True),
                                                               (BF, 128, 12, 2, 128, False, False), (BF, 128, 40, 40, 16, True, False)])
def test_append_many_tokens(dtype, Dh, Hq, Hkv, ps, major, adjacent):
    """Ragged prompts of so many tokens that a block takes several, whose groups straddle sequences."""
    new = (1, 2500, 3, 0, 1, 1700, 2)
    gg, rng = gen(17), np.random.default_rng(17)
    T, F = sum(new), Dh // 2
    table, pages = ref.table_for(rng, new, ps)
    kp, vp = (ref.pool(gg, 1, pages, Hkv, ps, Dh, dtype, major) for _ in "kv")
    cache = last.Cache(up(kp), up(vp))
    pos = torch.randint(0, 60000, (2, T), generator=gg, dtype=torch.int32)
    axis = np.arange(F) % 2
    rot = last.Rotary.make(freqs(F), axis=axis, adjacent=adjacent)
    q, k, v = (torch.randn((1, T, h, Dh), generator=gg).to(dtype) for h in (Hq, Hkv, Hkv))
    cu = np.concatenate([[0], np.cumsum(new)])
    got = last.rotary_append(rot, cache, last.Pages.make(table, new), pos.cuda(), q.cuda(), k.cuda(), v.cuda(), cu_new_h=cu)
    e = ref.rotary(q, pos, freqs(F), axis, adjacent)
    within(got, e, ref.rotary_bound(q, e, F, adjacent), "q")
    e = ref.rotary(k, pos, freqs(F), axis, adjacent)
    b = ref.rotary_bound(k, e, F, adjacent)
    exp_k, exp_v, tol = kp.double(), vp.clone(), torch.zeros(kp.shape, dtype=torch.float64)
    for r, n in enumerate(new):
        at = np.arange(n)
        page, slot = torch.from_numpy(table[r, at // ps].astype(np.int64)), torch.from_numpy(at % ps)
        rows = slice(int(cu[r]), int(cu[r + 1]))
        exp_k[0, page, :, slot], tol[0, page, :, slot], exp_v[0, page, :, slot] = e[0, rows], b[0, rows], v[0, rows]
    within(cache.k, exp_k, tol, "keys")
    assert same_bits(cache.v.cpu(), exp_v)


@pytest.mark.parametrize("dtype,Dh,Hkv,ps,major,G,R", [
    (BF, 128, 4, 16, False, 4, 9), (BF, 128, 2, 8, True, 3, 20), (F32, 128, 33, 16, False, 1, 3), (BF, 64, 1, 32, False, 5, 40),
    (F32, 64, 16, 64, True, 2, 6)])
def test_prune_batches(dtype, Dh, Hkv, ps, major, G, R):
    """So many rows that a block takes several layers, and heads so wide that it takes several turns."""
    gg, rng = gen(R), np.random.default_rng(R)
    N = rng.integers(1, 900, R)
    K = np.minimum(N, rng.integers(0, 400, R))
    vis, tail = rng.integers(0, 50, R), rng.integers(0, 60, R)
    lens, after = [int(x) for x in N + vis + tail], [int(x) for x in K + vis + tail]
    table, pages = ref.table_for(rng, lens + after, ps)
    src, dst = np.ascontiguousarray(table[:R]), np.ascontiguousarray(table[R:])
    kp, vp = (ref.pool(gg, G, pages, Hkv, ps, Dh, dtype, major) for _ in "kv")
    kept = [np.sort(rng.choice(n, k, replace=False)) for n, k in zip(N, K)]
    cu_vis, cu_keep = (np.concatenate([[0], np.cumsum(x)]) for x in (N, K))
    cache = last.Cache(up(kp), up(vp))
    flat = torch.from_numpy(np.concatenate(kept).astype(np.int32)).cuda()
    got = last.cache_prune(cache, last.Pages.make(src, lens), last.Pages.make(dst, after), vis, cu_vis, flat, cu_keep)
    assert got.tolist() == after
    for p, x in ((kp, cache.k), (vp, cache.v)):
        e = p.clone()
        for r in range(R):
            old = ref.prune_index(lens[r], int(vis[r]), int(N[r]), kept[r])
            i = np.arange(len(old))
            a, b, c, d = (torch.from_numpy(y.astype(np.int64)) for y in (src[r, old // ps], old % ps, dst[r, i // ps], i % ps))
            e[:, c, :, d] = p[:, a, :, b]
        assert same_bits(x.cpu(), e)


@pytest.mark.parametrize("dtype,Dh,Hkv,ps,major,G,n", [(BF, 128, 7, 16, False, 2, 301), (F32, 64, 2, 1024, True, 1, 20),
                                                       (BF, 64, 1, 8, False, 3, 1000)])
def test_copy_batches(dtype, Dh, Hkv, ps, major, G, n):
    gg, rng = gen(n), np.random.default_rng(n)
    kp, vp = (ref.pool(gg, G, 2 * n + 1, Hkv, ps, Dh, dtype, major) for _ in "kv")
    ids = rng.permutation(2 * n + 1)
    cache = last.Cache(up(kp), up(vp))
    last.cache_copy(cache, ids[:n], ids[n:2 * n])
    for p, got in ((kp, cache.k), (vp, cache.v)):
        e = p.clone()
        e[:, ids[n:2 * n]] = p[:, ids[:n]]
        assert same_bits(got.cpu(), e)


def test_nothing_to_do():
    """No tokens, no pages: nothing is launched, and nothing of the cache changes."""
    gg = gen(1)
    kp, vp = (ref.pool(gg, 2, 4, 2, 16, 64, BF) for _ in "kv")
    cache = last.Cache(kp.cuda(), vp.cuda())
    rot = last.Rotary.make(freqs(32))
    none = torch.empty((2, 0, 2, 64), dtype=BF, device="cuda")
    pos = torch.empty((1, 0), dtype=torch.int32, device="cuda")
    q, k = last.rotary(rot, pos, none, none)
    assert q.shape == k.shape == none.shape
    seqs = last.Pages.make([[0, 1], [2, 3]], [20, 0])
    assert last.rotary_append(rot, cache, seqs, pos, none, none, none, cu_new_h=[0, 0, 0]).shape == none.shape
    last.cache_copy(cache, [], [])
    empty = last.Pages.make([[0, 1], [2, 3]], [0, 0])
    got = last.cache_prune(cache, empty, last.Pages.make([[3], [2]], [0, 5]), [0, 0], [0, 0, 0],
                           torch.empty(0, dtype=torch.int32, device="cuda"), [0, 0, 0])
    assert got.tolist() == [0, 0]
    assert same_bits(cache.k.cpu(), kp) and same_bits(cache.v.cpu(), vp)


def test_prune_takes_any_indices():
    """Kept indices repeated and out of order are copied as they stand."""
    gg, ps = gen(2), 16
    kp, vp = (ref.pool(gg, 1, 12, 2, ps, 128, BF) for _ in "kv")
    cache = last.Cache(kp.cuda(), vp.cuda())
    src, dst = np.asarray([[7, 1, 4, 0]], np.int32), np.asarray([[9, 8]], np.int32)
    kept = np.asarray([30, 3, 3, 0, 39, 30, 30], np.int32)
    last.cache_prune(cache, last.Pages.make(src, [55]), last.Pages.make(dst, [22]), [5], [0, 40],
                     torch.from_numpy(kept).cuda(), [0, 7])
    old = [ref.prune_index(55, 5, 40, kept)]
    for p, x in ((kp, cache.k), (vp, cache.v)):
        assert same_bits(x.cpu(), ref.prune(p, src, dst, ps, old))


def test_two_calls_at_once():
    """Split calls on two streams, each with its own workspace, while a third stream copies pages of the cache."""
    lens = ((5000, 3, 800), (2000, 2000, 1))
    cases = [decode_case(51 + i, BF, 128, 28, 4, 16, n, G=1, layer=0) for i, n in enumerate(lens)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    qs = [c[2].cuda() for c in cases]
    used = set(cases[0][1].table_h[cases[0][1].table_h < 2 ** 30].tolist())
    free = [p for p in range(cases[0][0].k.shape[1]) if p not in used]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        last.cache_copy(cases[0][0], [int(cases[0][1].table_h[0, 0])], free[:1], stream=streams[2])
        for i, (c, q) in enumerate(zip(cases, qs)):
            got[i].append(last.decode_attention(c[0], c[1], q, stream=streams[i]))
    torch.cuda.synchronize()
    for (_, _, _, (out, _, ob, _)), g in zip(cases, got):
        for x in g:
            within(x, out, ob)
            assert same_bits(x, g[0])


def test_captured_prune_and_copy():
    """Prune and copy captured once and replayed on other contents, indices and lengths' targets, with eager work
    between the replays, equal the plain forms every time."""
    gg, rng, ps, G = gen(61), np.random.default_rng(61), 16, 2
    lens, vis, N, K = (200, 90), (7, 30), (150, 40), (33, 12)
    after = [n - a + b for n, a, b in zip(lens, N, K)]
    table, pages = ref.table_for(rng, list(lens) + after, ps)
    src, dst = np.ascontiguousarray(table[:2]), np.ascontiguousarray(table[2:])
    cu_vis, cu_keep = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (N, K))
    kd, vd = (torch.zeros((G, pages + 2, 2, ps, 128), dtype=BF, device="cuda") for _ in "kv")
    cache, full, into = last.Cache(kd, vd), last.Pages.make(src, lens), last.Pages.make(dst, after)
    kept = torch.zeros(sum(K), dtype=torch.int32, device="cuda")
    dev = [torch.from_numpy(np.asarray(x, np.int32)).cuda() for x in (vis, cu_vis, cu_keep, [src[0, 0], dst[1, 0]], [pages, pages + 1])]

    def step():
        last.cache_prune(cache, full, into, vis, cu_vis, kept, cu_keep, vis_start=dev[0], cu_vis=dev[1], cu_keep=dev[2])
        last.cache_copy(cache, [src[0, 0], dst[1, 0]], [pages, pages + 1], src=dev[3], dst=dev[4])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        kp, vp = (ref.pool(gg, G, pages + 2, 2, ps, 128, BF) for _ in "kv")
        kd.copy_(kp), vd.copy_(vp)
        ids = [np.sort(rng.choice(n, k, replace=False)) for n, k in zip(N, K)]
        kept.copy_(torch.from_numpy(np.concatenate(ids).astype(np.int32)))
        into.lens.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        assert into.lens.tolist() == after
        old = [ref.prune_index(lens[r], vis[r], N[r], ids[r]) for r in range(2)]
        for p, x in ((kp, kd), (vp, vd)):
            e = ref.prune(p, src, dst, ps, old)
            e[:, pages], e[:, pages + 1] = e[:, src[0, 0]], e[:, dst[1, 0]]
            assert same_bits(x.cpu(), e)


@pytest.mark.parametrize("bound", [2048, 8192])
def test_decode_one_long_among_short(bound):
    """Bounds that say nothing of the lengths: one sequence as long as they allow, the others short."""
    R, ps, Hkv, Dh = 64, 64, 4, 128
    gg, rng = gen(9), np.random.default_rng(9)
    lens = rng.integers(0, 300, R)
    lens[41] = bound
    pages = 200
    table = rng.integers(0, pages, (R, bound // ps)).astype(np.int32)      # pages may be shared: they are only read
    kp, vp = (ref.pool(gg, 1, pages, Hkv, ps, Dh, BF) for _ in "kv")
    q = torch.randn((R, 28, Dh), generator=gg).to(BF)
    seqs = last.Pages(lens_h=np.full(R, bound), table=torch.from_numpy(table).cuda(),
                      lens=torch.from_numpy(lens.astype(np.int32)).cuda())
    check(last.Cache(kp.cuda(), vp.cuda()), seqs, q, ref.decode(q, kp[0], vp[0], table, lens), lens, 0)
