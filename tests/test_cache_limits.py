"""Calls at the limits of what one launch holds, without a GPU where they are refused on the host: nothing they
were given is followed or written."""
import numpy as np
import pytest

from paper_2607_27952_amd import last
from test_cache_abi import UNS, Call


@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 31 - 4, 2 ** 30])
@pytest.mark.parametrize("Hq,Hkv,Dh,G", [(1, 0, 64, 1), (1, 1, 128, 1), (0, 1, 64, 2), (64, 8, 128, 1)])
def test_rotary_refuses_the_most_tokens(T, Hq, Hkv, Dh, G):
    """More tokens than a launch holds, up to the largest number of them."""
    c = Call()
    c.a.update(G=G, T=T, Hq=Hq, Hkv=Hkv, Dh=Dh)
    c.rot.n_axes = 1
    row = max(Hq, Hkv) * Dh
    for n in ("q", "k"):
        c.heads[n] = last._Heads(c.mem["q"].p, 0, 0)
    for n in ("q_out", "k_out"):
        c.heads[n] = last._Heads(c.mem["out"].p, row * T, row)
    assert c.rotary() == UNS and c.untouched()


@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 4])
def test_append_refuses_the_most_tokens(T):
    c = Call()
    c.a.update(G=1, T=T, Hq=0)
    c.cu_new[:] = [0, 1, T]
    for n in ("k", "v"):
        c.heads[n] = last._Heads(c.mem["q"].p, 0, 0)
    assert c.append() == UNS and c.untouched()


def test_prune_refuses_more_tiles_than_a_launch_holds():
    """2^14 sequences whose longest new length is 2^15: 2^24 blocks of 32 tokens, whatever the others keep."""
    R, n = 1 << 14, 1 << 15
    c = Call()
    c.cache.page_size, c.cache.head_stride, c.cache.page_stride = 1024, 1024 * 64, 4 * 1024 * 64
    c.cache.n_pages = 32 + R + 32
    c.cache.layer_stride = c.cache.n_pages * c.cache.page_stride
    c.lens, c.later = np.full(R, 40, np.int32), np.full(R, 40, np.int32)
    c.lens[3] = c.later[3] = n
    c.table = np.tile(np.arange(32, dtype=np.int32), (R, 1))
    c.into = np.zeros((R, 32), np.int32)
    c.into[:, 0] = 64 + np.arange(R)
    c.into[3] = 32 + np.arange(32)
    for p, table, lens in ((c.pages, c.table, c.lens), (c.dst, c.into, c.later)):
        p.R, p.max_pages, p.table_h, p.lens_h = R, 32, table.ctypes.data, lens.ctypes.data
    c.vis, c.cu_vis, c.cu_keep = np.zeros(R, np.int32), np.zeros(R + 1, np.int32), np.zeros(R + 1, np.int32)
    assert c.prune() == UNS and c.untouched()


def test_copy_refuses_more_pieces_than_a_launch_holds():
    """Pages of 512 KB a layer: 2 layers of 32768 pages are 64 GiB."""
    c = Call()
    c.cache.page_size, c.cache.head_stride, c.cache.page_stride = 1024, 1024 * 64, 4 * 1024 * 64
    n = 1 << 15
    c.cache.n_pages = 2 * n
    c.cache.layer_stride = c.cache.n_pages * c.cache.page_stride
    ids = np.arange(2 * n, dtype=np.int32)
    c.src_h, c.dst_h, c.a["n"] = ids[:n].copy(), ids[n:].copy(), n
    assert c.copy() == UNS and c.untouched()
    c.cache.page_size, c.cache.Hkv, c.a["n"] = 512, 1 << 16, 1            # and a page of 2^25 rows
    c.cache.head_stride, c.cache.page_stride = 512 * 64, 512 * 64 << 16
    c.cache.layer_stride = c.cache.n_pages * c.cache.page_stride
    assert c.copy() == UNS and c.untouched()


def decode_limits(R, Hkv, Hq, bound):
    c = Call()
    c.cache.Hkv, c.cache.page_size, c.cache.head_stride, c.cache.page_stride = Hkv, 1024, 1024 * 64, Hkv * 1024 * 64
    c.cache.layer_stride = c.cache.n_pages * c.cache.page_stride
    c.lens = np.full(R, bound, np.int32)
    c.pages.R, c.pages.max_pages, c.pages.table_h, c.pages.lens_h = R, max(1, bound // 1024), None, c.lens.ctypes.data
    c.a["Hq"], c.a["q_stride"] = Hq, Hq * 64
    return c


@pytest.mark.parametrize("R,Hkv,Hq,bound", [(1 << 18, 64, 64, 1), (1 << 17, 64, 64, 1 << 19), (1 << 8, 1 << 14, 1 << 14, 1)])
def test_decode_refuses_more_than_a_launch_holds(R, Hkv, Hq, bound):
    """2^24 query heads, 2^23 of them with 4096 steps and more each, 2^22 units."""
    c = decode_limits(R, Hkv, Hq, bound)
    assert c.decode() == UNS and c.untouched()
    assert last.lib().last_decode_attention_workspace(c.cache, c.pages, Hq) == 0


def test_decode_takes_what_is_always_taken():
    """Just under the bounds that are always taken: the query answers."""
    for R, Hkv, Hq, bound in (((1 << 16) - 1, 1, 64, 1 << 13), (1 << 10, 4, 4, 1 << 22), ((1 << 22) - 1, 1, 1, 1 << 13)):
        c = decode_limits(R, Hkv, Hq, bound)
        assert R * Hq < 2 ** 22 and R * Hq * bound < 2 ** 35
        assert last.lib().last_decode_attention_workspace(c.cache, c.pages, Hq) >= 256
