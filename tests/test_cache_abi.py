"""What the calls of the rotation and the paged cache refuse, without a GPU: every malformed call is
turned away on the host before any HIP call, and nothing it was given is written."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2607_27952_amd import last

OK, INV, UNS, WS = last.LAST_OK, last.LAST_ERR_INVALID, last.LAST_ERR_UNSUPPORTED, last.LAST_ERR_WORKSPACE


class Fake:
    """A host buffer standing in for device memory; a refused call never follows it."""

    def __init__(self, n=1 << 12):
        self.buf = np.full(n + 64, 0x5A5A5A5A, np.uint32)
        self.p = (self.buf.ctypes.data + 255) // 256 * 256

    def untouched(self):
        return bool(np.all(self.buf == 0x5A5A5A5A))


class Call:
    """A valid call's arguments (2 sequences, 2 layers, 4 heads of 64, pages of 16), to be spoilt one at a time."""

    def __init__(self, dtype=last.LAST_BF16):
        self.mem = {n: Fake() for n in ("k", "v", "q", "out", "ws", "dev", "lens")}
        m = self.mem
        self.cache = last._Cache(2, 20, 16, 4, 64, dtype, 20 * 4 * 16 * 64, 4 * 16 * 64, 16 * 64, 64, m["k"].p, m["v"].p)
        self.table = np.arange(6, dtype=np.int32).reshape(2, 3).copy()
        self.into = np.arange(10, 16, dtype=np.int32).reshape(2, 3).copy()
        self.lens = np.asarray([40, 17], np.int32)
        self.later = np.asarray([40, 40], np.int32)
        self.pages = last._Pages(2, 3, m["dev"].p, self.table.ctypes.data, m["lens"].p, self.lens.ctypes.data)
        self.dst = last._Pages(2, 3, m["dev"].p, self.into.ctypes.data, m["dev"].p, self.later.ctypes.data)
        self.axis = np.zeros(32, np.int32)
        self.rot = last._Rotation(3, 32, 0, 0, m["dev"].p, m["dev"].p, self.axis.ctypes.data)
        self.heads = {n: last._Heads(m["q"].p, 2 * 512, 512) for n in ("q", "k", "v", "q_out", "k_out")}
        self.vis, self.cu_vis, self.cu_keep = (np.asarray(a, np.int32) for a in ([4, 2], [0, 20, 30], [0, 3, 5]))
        self.cu_new = np.asarray([0, 1, 2], np.int32)
        self.a = {"dtype": dtype, "G": 2, "T": 2, "Hq": 8, "Hkv": 4, "Dh": 64, "layer": 0, "pos": m["dev"].p, "scale": 0.0,
                  "q": m["q"].p, "q_stride": 512, "out": m["out"].p, "lse": None, "ws": m["ws"].p, "ws_bytes": 1 << 14,
                  "cu_new": m["dev"].p, "n": 3, "kept": m["dev"].p, "new_lens": m["out"].p}
        self.src_h, self.dst_h = np.asarray([0, 1, 1], np.int32), np.asarray([5, 7, 6], np.int32)

    def rotary(self):
        a, h = self.a, self.heads
        return last.lib().last_rotary(self.rot, a["dtype"], a["G"], a["T"], a["Hq"], a["Hkv"], a["Dh"], a["pos"], h["q"], h["k"],
                                      h["q_out"], h["k_out"], None)

    def append(self):
        a, h = self.a, self.heads
        return last.lib().last_rotary_append(self.rot, self.cache, a["layer"], a["G"], self.pages, a["T"], a["cu_new"],
                                             None if self.cu_new is None else self.cu_new.ctypes.data, a["Hq"], a["pos"],
                                             h["q"], h["q_out"], h["k"], h["v"], None)

    def decode(self):
        a = self.a
        return last.lib().last_decode_attention(self.cache, a["layer"], self.pages, a["Hq"], a["scale"], a["q"], a["q_stride"],
                                                a["out"], a["lse"], a["ws"], a["ws_bytes"], None)

    def prune(self):
        a, d = self.a, self.mem["dev"].p
        return last.lib().last_cache_prune(self.cache, self.pages, self.dst, d, self.vis.ctypes.data, d, self.cu_vis.ctypes.data,
                                           a["kept"], d, self.cu_keep.ctypes.data, a["new_lens"], None)

    def copy(self):
        a, d = self.a, self.mem["dev"].p
        return last.lib().last_cache_copy(self.cache, a["n"], d, self.src_h.ctypes.data, d, self.dst_h.ctypes.data, None)

    def untouched(self):
        return all(f.untouched() for f in self.mem.values())


def spoil(c, where, value):
    at, key = where.split(".")
    box = getattr(c, at)
    if isinstance(box, dict):
        box[key] = value
    elif isinstance(box, np.ndarray):
        box.reshape(-1)[int(key)] = value
    else:
        setattr(box, key, value)


CACHE = [("cache.G", 0, INV), ("cache.n_pages", 0, INV), ("cache.page_size", 12, UNS), ("cache.page_size", 4, UNS),
         ("cache.page_size", 2048, UNS), ("cache.Dh", 96, UNS), ("cache.Hkv", 0, INV), ("cache.dtype", 5, INV),
         ("cache.token_stride", 32, INV), ("cache.token_stride", 66, INV), ("cache.head_stride", 512, INV),
         ("cache.page_stride", 16 * 64, INV), ("cache.layer_stride", -4096, INV), ("cache.layer_stride", 1 << 50, INV),
         ("cache.k", None, INV)]
PAGES = [("pages.R", 0, INV), ("pages.max_pages", 0, INV), ("pages.table", None, INV), ("pages.lens", None, INV),
         ("pages.lens_h", None, INV), ("lens.0", 49, INV), ("lens.1", -1, INV), ("table.4", 20, INV), ("table.0", -1, INV),
         ("pages.max_pages", 1 << 27, UNS)]
ROT = [("rot.n_axes", 0, INV), ("rot.n_axes", 5, UNS), ("rot.n_freqs", 0, INV), ("rot.n_freqs", 40, INV), ("rot.n_freqs", 12, UNS),
       ("rot.inv_freq", None, INV), ("rot.axis", None, INV), ("rot.axis_h", None, INV), ("axis.31", 3, INV), ("axis.0", -1, INV)]


@pytest.mark.parametrize("where,value,status", ROT + [
    ("a.dtype", 3, INV), ("a.G", 0, INV), ("a.T", -1, INV), ("a.Hq", -1, INV), ("a.Dh", 0, INV), ("a.Dh", 32, UNS), ("a.Dh", 80, UNS), ("a.pos", None, INV),
    ("heads.q", None, INV), ("heads.k_out", None, INV)])
def test_rotary_refuses(where, value, status):
    c = Call()
    spoil(c, where, value)
    assert c.rotary() == status and c.untouched()


@pytest.mark.parametrize("which,data,layer,token", [
    ("q", 8, 1024, 512), ("q", 0, 1024, 516), ("q", 0, 1020, 512), ("q", 0, 1024, -512), ("q_out", 0, 1024, 0), ("q_out", 0, 0, 512),
    ("q_out", 0, 512, 512), ("k_out", 0, 512, 128), ("q_out", 0, 2048, 1024), ("k", 0, 1 << 49, 512)])
def test_rotary_refuses_rows(which, data, layer, token):
    """Rows off 16 bytes, strides off 16 bytes or negative, written rows on top of each other, and turned in
    place with other strides than read (the last q_out; q is read at 512)."""
    c = Call()
    c.heads[which] = last._Heads(c.mem["q"].p + data, layer, token)
    assert c.rotary() == INV and c.untouched()


@pytest.mark.parametrize("where,value,status", CACHE + PAGES + ROT + [
    ("a.layer", -1, INV), ("a.layer", 1, INV), ("a.G", 3, INV), ("a.T", 3, INV), ("a.Hq", -1, INV), ("a.pos", None, INV),
    ("a.cu_new", None, INV), ("cu_new.1", 3, INV), ("cu_new.0", 1, INV), ("heads.k", None, INV), ("heads.v", None, INV),
    ("heads.q_out", None, INV)])
def test_append_refuses(where, value, status):
    c = Call()
    c.rot.n_freqs = 32
    spoil(c, where, value)
    assert c.append() == status and c.untouched()


def test_append_refuses_queries_without_a_rotation_and_other_counts():
    c = Call()
    c.rot = None
    assert c.append() == INV
    c = Call()
    c.a["cu_new"], c.cu_new, c.a["T"] = None, None, 3      # one token per sequence, but three tokens
    assert c.append() == INV and c.untouched()
    c = Call()
    c.a["T"], c.cu_new[:] = 0, 0
    assert c.append() == OK and c.untouched()               # no token: nothing to do


@pytest.mark.parametrize("where,value,status", CACHE + PAGES + [
    ("a.layer", 2, INV), ("a.layer", -1, INV), ("a.Hq", 6, INV), ("a.Hq", 0, INV), ("a.scale", float("nan"), INV), ("a.q", None, INV),
    ("a.out", None, INV), ("a.q_stride", -512, INV), ("a.q_stride", 508, INV), ("a.lse", 2, INV), ("a.ws", None, WS),
    ("a.ws_bytes", 255, WS)])
def test_decode_refuses(where, value, status):
    c = Call()
    spoil(c, where, value)
    assert c.decode() == status and c.untouched()


def test_decode_workspace():
    c = Call()
    L = last.lib()
    assert L.last_decode_attention_workspace(c.cache, c.pages, 8) >= 256
    assert L.last_decode_attention_workspace(c.cache, c.pages, 6) == 0
    c.a["ws"] += 64
    assert c.decode() == WS and c.untouched()
    c = Call()
    c.a["q"] += 8
    assert c.decode() == INV and c.untouched()


@pytest.mark.parametrize("where,value,status", CACHE + PAGES + [
    ("pages.table_h", None, INV), ("dst.table_h", None, INV), ("dst.lens_h", None, INV), ("dst.R", 1, INV), ("later.0", 22, INV),
    ("into.1", 20, INV), ("into.1", 10, INV), ("into.3", 11, INV), ("into.0", 4, INV), ("into.4", 0, INV), ("vis.0", -1, INV),
    ("vis.1", 8, INV), ("cu_vis.1", 40, INV), ("cu_keep.1", 21, INV), ("cu_keep.0", 1, INV), ("a.kept", None, INV)])
def test_prune_refuses(where, value, status):
    """Among them target pages named twice or by the source: 23 of 40 and 9 of 17 tokens stay, in two pages and one."""
    c = Call()
    spoil(c, where, value)
    if where in ("into.4",):
        c.later[1] = 17
        c.vis[1], c.cu_keep[2] = 2, 3 + 10                   # all 17 tokens stay, in two pages
        c.cu_keep[1] = 3
    assert c.prune() == status and c.untouched()


def test_prune_refuses_its_own_lengths_and_late_sharing():
    c = Call()
    c.a["new_lens"] = c.mem["lens"].p
    assert c.prune() == INV and c.untouched()
    c = Call()
    c.into[0, 0] = c.table[0, 0]                             # token 4 of that page is already a visual one
    assert c.prune() == INV and c.untouched()


@pytest.mark.parametrize("where,value,status", CACHE + [
    ("a.n", -1, INV), ("src_h.0", -1, INV), ("src_h.2", 20, INV), ("dst_h.1", 20, INV), ("dst_h.1", 5, INV), ("dst_h.0", 1, INV),
    ("src_h.0", 6, INV)])
def test_copy_refuses(where, value, status):
    c = Call()
    spoil(c, where, value)
    assert c.copy() == status and c.untouched()
    c = Call()
    c.a["n"] = 0
    assert c.copy() == OK and c.untouched()


def test_cache_refuses_one_buffer_for_keys_and_values():
    c = Call()
    c.cache.v = c.cache.k
    assert c.decode() == INV and c.untouched()


def test_binding_refuses():
    k, v = torch.zeros(2, 3, 4, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 3, 4, 16, 64, dtype=torch.bfloat16)
    last.Cache(k, v)
    for a, b in ((k[0], v[0]), (k, v[:1]), (k, v.transpose(2, 3).contiguous().transpose(2, 3)), (k, v.float()),
                 (k.transpose(3, 4), v.transpose(3, 4))):
        with pytest.raises((ValueError, TypeError)):
            last.Cache(a, b)
    with pytest.raises(TypeError):
        last.Cache(k.half(), v.half())
    t, n = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    last.Pages(lens_h=[0, 0], table=t, lens=n)
    for kw in ({"table": t[0]}, {"table": t.long()}, {"lens": n[:1]}, {"lens_h": [0]}, {"table_h": np.zeros((2, 2))},
               {"table": t.t().contiguous().t()}):
        with pytest.raises(ValueError):
            last.Pages(**{"lens_h": [0, 0], "table": t, "lens": n, **kw})
    with pytest.raises(ValueError):
        last.Rotary.make(np.ones(8), sections=(3, 4), device="cpu")
    rot = last.Rotary.make(np.ones(32), sections=(8, 24), device="cpu")
    assert rot.n_axes == 2 and rot.axis_h.tolist() == [0] * 8 + [1] * 24
    q = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        last.rotary(rot, torch.zeros(2, 2, dtype=torch.int32), q)          # not on a GPU
    with pytest.raises(ValueError):
        last.decode_attention(last.Cache(k, v), last.Pages.make(t, n, device="cpu"), q[0])
