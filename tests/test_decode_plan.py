"""How decode attention lays a call out by the bounds of its lengths: the workspace it asks for, and when it splits."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2607_27952_amd import last


class Asked:
    """The workspace query with made-up addresses: it follows none of them on the device."""

    def __init__(self, dtype, Hkv, Hq, Dh, major, max_pages=8192):
        ps, self.Hq, self.max_pages = 16, Hq, max_pages
        hs, ts = (Dh, Hkv * Dh) if major else (ps * Dh, Dh)
        page = Hkv * ps * Dh
        self.cache = last._Cache(1, 64, ps, Hkv, Dh, dtype, 64 * page, page, hs, ts, 1 << 20, 1 << 21)

    def bytes(self, lens):
        lens = np.ascontiguousarray(lens, dtype=np.int32)
        pages = last._Pages(len(lens), self.max_pages, 256, None, 256, lens.ctypes.data)
        return last.lib().last_decode_attention_workspace(self.cache, pages, self.Hq)


SHAPES = [(last.LAST_BF16, 32, 32, 128, False), (last.LAST_BF16, 4, 28, 128, True), (last.LAST_BF16, 8, 32, 64, False),
          (last.LAST_F32, 16, 16, 64, True), (last.LAST_BF16, 1, 40, 128, False)]


@pytest.mark.parametrize("shape", SHAPES)
def test_workspace_covers_shorter_bounds(shape):
    """A workspace for some bounds serves every call whose bounds are no longer, and of no more sequences."""
    ask, rng = Asked(*shape), np.random.default_rng(3)
    assert ask.bytes([0]) >= 256
    for R, longest in ((64, 2048), (64, 640), (32, 1000), (1, 104), (200, 16), (8, 100000), (256, 3)):
        for _ in range(30):
            lens = np.full(R, longest) if rng.random() < 0.5 else rng.integers(0, longest + 1, R)
            need = ask.bytes(lens)
            shorter = [np.minimum(lens, rng.integers(0, longest + 1, R)), np.minimum(lens, rng.integers(0, longest + 1)), lens // 64,
                       np.where(np.arange(R) < max(1, R // 16), lens, 10), np.where(rng.random(R) < 0.1, lens, 0)]
            for less in shorter:
                less = np.minimum(less, lens)
                assert ask.bytes(less) <= need, (R, longest)
                assert ask.bytes(less[:rng.integers(1, R + 1)]) <= need, (R, longest)


@pytest.mark.gpu
@pytest.mark.parametrize("longest,short", [(640, 10), (2048, 100)])
def test_workspace_of_the_longest_bounds_serves_shorter_ones(longest, short):
    """One workspace, sized once for even long bounds, in calls of ragged shorter ones."""
    R, Hkv, Hq, Dh, ps = 64, 4, 28, 128, 16
    gg, rng = torch.Generator().manual_seed(2), np.random.default_rng(2)
    kp, vp = (ref.pool(gg, 1, 256, Hkv, ps, Dh, torch.bfloat16) for _ in "kv")
    cache = last.Cache(kp.cuda(), vp.cuda())
    table = rng.integers(0, 256, (R, longest // ps)).astype(np.int32)       # pages are only read: they may be shared
    need = last.decode_attention_workspace(cache, last.Pages.make(table, [longest] * R), Hq)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    q = torch.randn((R, Hq, Dh), generator=gg).bfloat16()
    for lens in ([longest] * 4 + [short] * 60, [longest] + [0] * 63, [short] * 64, [longest] * 64):
        got = last.decode_attention(cache, last.Pages.make(table, lens), q.cuda(), ws=ws).cpu().double()
        out, _, bound, _ = ref.decode(q, kp[0], vp[0], table, lens)
        assert bool(((got - out).abs() <= bound).all())


def kernels_of(call):
    last.profile_enable(True)
    try:
        torch.cuda.synchronize()
        last.profile_collect()
        last.profile_reset()
        got = call()
        torch.cuda.synchronize()
        return got, {name: n for name, (n, _) in last.profile_collect().items() if n}
    finally:
        last.profile_enable(False)


@pytest.mark.gpu
@pytest.mark.parametrize("R,longest,at", [(256, 6000, 77), (200, 20000, 0), (64, 2100, 63)])
def test_a_long_sequence_among_empty_slots_is_split(R, longest, at):
    """A padded batch whose empty slots have bounds of 0: its one long sequence is shared out among the blocks."""
    Hkv, Hq, Dh, ps = 2, 8, 128, 16
    gg, rng = torch.Generator().manual_seed(4), np.random.default_rng(4)
    lens = np.zeros(R, np.int32)
    lens[at] = longest
    kp, vp = (ref.pool(gg, 1, 128, Hkv, ps, Dh, torch.bfloat16) for _ in "kv")
    table = rng.integers(0, 128, (R, -(-longest // ps))).astype(np.int32)
    q = torch.randn((R, Hq, Dh), generator=gg).bfloat16()
    cache, pages = last.Cache(kp.cuda(), vp.cuda()), last.Pages.make(table, lens)
    got, kernels = kernels_of(lambda: last.decode_attention(cache, pages, q.cuda(), want_lse=True))
    assert kernels == {"decode": 1, "decode_join": 1}
    out, lse, bound, lbound = ref.decode(q, kp[0], vp[0], table, lens)
    assert bool(((got[0].cpu().double() - out).abs() <= bound).all())
    assert float((got[1][at].cpu().double() - lse[at]).abs().max()) <= float(lbound[at].max())
    rest = np.arange(R) != at
    assert bool((got[0][rest] == 0).all()) and bool((got[1][rest] == -float("inf")).all())


@pytest.mark.gpu
def test_lengths_are_cut_to_the_longest_bound():
    """A length above its own sequence's bound is taken up to the longest bound of the call, by decode and append."""
    Hkv, Dh, ps = 2, 64, 16
    gg = torch.Generator().manual_seed(6)
    kp, vp = (ref.pool(gg, 1, 24, Hkv, ps, Dh, torch.bfloat16) for _ in "kv")
    table = np.arange(21, dtype=np.int32).reshape(3, 7)
    q = torch.randn((3, 4, Dh), generator=gg).bfloat16()
    cache = last.Cache(kp.cuda(), vp.cuda())
    pages = last.Pages(lens_h=np.asarray([40, 100, 0]), table=torch.from_numpy(table).cuda(),
                       lens=torch.tensor([70, 112, 1], dtype=torch.int32, device="cuda"))
    got = last.decode_attention(cache, pages, q.cuda()).cpu().double()
    out, _, bound, _ = ref.decode(q, kp[0], vp[0], table, (70, 100, 1))
    assert bool(((got - out).abs() <= bound).all())
    k, v = (torch.randn((1, 3, Hkv, Dh), generator=gg).bfloat16() for _ in "kv")
    last.rotary_append(None, cache, pages, None, None, k.cuda(), v.cuda())
    for pool, x, now in ((kp, k, cache.k), (vp, v, cache.v)):
        pool[0, 4, :, 5], pool[0, 14, :, 0] = x[0, 0], x[0, 2]      # tokens 69 and 0; 111 lies behind the longest bound
        assert torch.equal(now.cpu().view(torch.int16), pool.view(torch.int16))
