"""Calls at the limits of what one launch holds, without a GPU where they are refused on the host: nothing they
were given is followed or written."""
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
