"""Prune where many sequences are short and one is long, so that tiles counted by the longest would not fit a
launch (needs an MI355X)."""
import numpy as np
import pytest
import torch

from paper_2607_27952_amd import last

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Dh,Hkv,G,R,longest,ps", [
    (torch.bfloat16, 64, 32, 8, 6000, 1500, 8),     # 2 tokens and 2 pools a block by the rule: 36 million blocks
    (torch.float32, 128, 2, 1, 8000, 60000, 64)])   # 4 tokens and both pools: 120 million, so that tiles grow too
def test_prune_one_long_sequence_among_short_ones(dtype, Dh, Hkv, G, R, longest, ps):
    at = R // 3
    N, text = longest // 2, longest // 2 + 100      # the long one: half its visual tokens go
    K = N - 100
    lens = np.full(R, 5, np.int32)
    lens[at] = N + text
    after = lens.copy()
    after[at] = K + text
    n_src, n_dst = -(-lens[at] // ps), -(-after[at] // ps)
    short = n_src + n_dst                           # one page read by all short sequences, then a page each
    src, dst = np.zeros((R, n_src), np.int32), np.zeros((R, n_dst), np.int32)
    src[:, 0], dst[:, 0] = short, short + 1 + np.arange(R)
    rng = np.random.default_rng(1)
    ids = rng.permutation(short)
    src[at], dst[at] = ids[:n_src], ids[n_src:]
    shape = (G, short + 1 + R, ps, Hkv, Dh)         # the heads of a token together
    gg = torch.Generator(device="cuda").manual_seed(1)
    pools = []
    for _ in "kv":
        pool = torch.zeros(shape, dtype=dtype, device="cuda")
        pool[:, :short + 1] = torch.randn((G, short + 1) + shape[2:], generator=gg, device="cuda").to(dtype)
        pools.append(pool)
    before = [p[:, :short + 1].clone() for p in pools]
    vis, n_vis, n_keep = np.zeros(R, np.int32), np.zeros(R, np.int32), np.zeros(R, np.int32)
    vis[at], n_vis[at], n_keep[at] = 50, N, K
    vis[0], n_vis[0], n_keep[0] = 1, 3, 1           # a short one loses two of its tokens
    after[0] = 3
    kept = np.concatenate([[2], np.sort(rng.choice(N, K, replace=False))]).astype(np.int32)
    cu = lambda x: np.concatenate([[0], np.cumsum(x)]).astype(np.int32)
    into = last.Pages.make(dst, after)
    got = last.cache_prune(last.Cache(*(p.transpose(2, 3) for p in pools)), last.Pages.make(src, lens), into, vis, cu(n_vis),
                           torch.from_numpy(kept).cuda(), cu(n_keep))
    assert got.tolist() == after.tolist()
    old = np.concatenate([np.arange(50), 50 + kept[1:], np.arange(50 + N, lens[at])])
    new = np.arange(len(old))
    a, b, x, y = (torch.from_numpy(i.astype(np.int64)).cuda() for i in (src[at, old // ps], old % ps, dst[at, new // ps], new % ps))
    kind = torch.int16 if dtype == torch.bfloat16 else torch.int32
    for p, was in zip(pools, before):
        now, was = p.view(kind), was.view(kind)
        assert torch.equal(now[:, x, y], was[:, a, b])
        assert torch.equal(now[:, src[at]], was[:, src[at]])                      # the source stays whole
        pages = now[:, short + 1:]
        five = was[:, short:short + 1, :5]
        assert bool((pages[:, 1:at, :5] == five).all()) and bool((pages[:, at + 1:, :5] == five).all())
        assert torch.equal(pages[:, 0, :3], five[:, 0, [0, 3, 4]])                # token 1 + kept 2, then the rest
        assert not bool(pages[:, 0, 3:].any()) and not bool(pages[:, 1:, 5:].any()) and not bool(pages[:, at].any())
