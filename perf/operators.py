"""The paged cache and what writes, reads, prunes and copies it, as cases with
inputs, a call and a 64-bit result each.

A case is a dict of plain values; ``op`` names the public call:

  rotary   last_rotary: queries and keys turned by positions with one or
           three axes; ``inverse`` is the gradient's direction
  append   last_rotary_append: the same, the keys and values written into the
           pages of a cache
  decode   last_decode_attention: one new token per sequence over its pages
  prune    last_cache_prune: the cache of a full prompt compacted to its text
           and the visual tokens that were kept
  copy     last_cache_copy: pages copied in every layer

A cache holds G layers of keys and values in pages of ``page`` tokens,
[G][pages][Hkv][page][Dh], or with ``token_major`` [G][pages][page][Hkv][Dh].
Where ``hi`` is above ``lo`` the sequences are ragged, their lengths drawn
log-uniform from ``sizes``. Pages lie in the pool in random order.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# (Hq, Hkv, Dh, dtype): the head shapes of the workloads
SHAPES = ((16, 16, 64, "f32"), (32, 32, 128, "bf16"), (32, 8, 128, "bf16"), (12, 2, 128, "bf16"), (28, 4, 128, "bf16"))

#: The most bytes a drawn case of each call moves: what its largest listed one does.
MOST = {"rotary": 2.1e9, "append": 1.3e9, "decode": 0.6e9, "prune": 0.5e9, "copy": 1.0e9}


def _case(name, op, shape, **more):
    c = {"op": op, "Hq": shape[0], "Hkv": shape[1], "Dh": shape[2], "dtype": shape[3], **more}
    if name:
        c["name"] = name
    return c


def _rotary(name, shape, T, G=1, axes=3, rot=None, adjacent=False, inverse=False, far=0):
    return _case(name, "rotary", shape, T=T, G=G, axes=axes, rot=rot or shape[2], adjacent=adjacent, inverse=inverse, far=far)


def _append(name, shape, R, new, past, G=1, axes=3, rot=None, adjacent=False, page=16, token_major=False, sizes=1):
    return _case(name, "append", shape, R=R, G=G, axes=axes, rot=rot or shape[2], adjacent=adjacent, page=page,
                 token_major=token_major, lo=new[0], hi=new[1], past_lo=past[0], past_hi=past[1], sizes=sizes)


def _decode(name, shape, R, lens, page=16, token_major=False, sizes=1):
    return _case(name, "decode", shape, R=R, G=1, page=page, token_major=token_major, lo=lens[0], hi=lens[1], sizes=sizes)


def _prune(name, shape, R, G, n, text, keep, page=16, token_major=False, sizes=1):
    return _case(name, "prune", shape, R=R, G=G, page=page, token_major=token_major, lo=n[0], hi=n[1], text_lo=text[0],
                 text_hi=text[1], keep_num=keep[0], keep_den=keep[1], sizes=sizes)


def _copy(name, shape, n, G, page=16, token_major=False):
    return _case(name, "copy", shape, n=n, G=G, page=page, token_major=token_major)


def listed():
    return [
        # The gradient of the rotation on a serving batch's prompt: 64 images of 576 tokens with 64 text tokens each.
        _rotary("rotary_gradient_batch", SHAPES[1], 64 * 640, axes=1, inverse=True),
        # Queries and keys of one layer of the prefill of eight 64-frame videos, positions in time, height and width.
        _rotary("rotary_video", SHAPES[4], 8 * 16512),
        # One decoding step of 64 requests: every request's new token turned and put into its page.
        _append("append_step", SHAPES[1], 64, (1, 1), (639, 639), axes=1),
        # A ragged batch of dynamic-resolution prompts put into a cache, 288 to 16640 tokens each.
        _append("append_dynres", SHAPES[3], 32, (288, 16640), (0, 0)),
        # One request on its own in fp32, after its 576 visual tokens were pruned to 64.
        _decode("decode_one_fp32", SHAPES[0], 1, (104, 104)),
        # The serving batch of 64 requests with all their tokens, one KV head a query head.
        _decode("decode_llava_batch", SHAPES[1], 64, (640, 640)),
        # The ragged batch of dynamic-resolution prompts, 12 query heads on 2 KV heads.
        _decode("decode_dynres", SHAPES[3], 128, (288, 16640)),
        # Eight videos: few sequences, long ones, grouped-query heads.
        _decode("decode_video", SHAPES[4], 8, (16512, 16512), page=64, token_major=True),
        # The serving batch pruned to one ninth of its visual tokens, two layers.
        _prune("prune_llava_batch", SHAPES[1], 64, 2, (576, 576), (64, 64), (1, 9)),
        # Eight videos pruned to one sixteenth, four layers of grouped-query heads.
        _prune("prune_video", SHAPES[4], 8, 4, (16384, 16384), (128, 128), (1, 16), page=64, token_major=True),
        # Eight continuations of one request: the last page of each, in four layers.
        _copy("copy_fork", SHAPES[4], 8, 4),
        # Many pages moved at once.
        _copy("copy_many", SHAPES[2], 1024, 2, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "append", "decode", "decode", "decode", "prune", "copy"))
    shape = rng.choice(SHAPES)
    Hq, Hkv, Dh, dtype = shape
    e = 4 if dtype == "f32" else 2
    page = rng.choice((8, 16, 32, 64, 128, 256))
    major = rng.random() < 0.5
    sizes = rng.randrange(1 << 20)
    axes, rot, adjacent = rng.choice((1, 3)), rng.choice((Dh, Dh, Dh // 2)), rng.random() < 0.3
    if op == "rotary":
        G = rng.choice((1, 1, 2, 4))
        T = _log(rng, 1, MOST[op] / (2 * G * (Hq + Hkv) * Dh * e))
        return _rotary(None, shape, T, G, axes, rot, adjacent, rng.random() < 0.4, rng.choice((0, 0, 1 << 20)))
    if op == "append":
        G = rng.choice((1, 1, 2))
        most = MOST[op] / (2 * G * (Hq + 2 * Hkv) * Dh * e)
        R = _log(rng, 1, 128)
        if rng.random() < 0.4:
            new = (1, 1)
        else:
            hi = _log(rng, 2, max(2, min(16640, most / R)))
            new = (max(1, hi // rng.choice((1, 4, 16))), hi)
        past = rng.choice(((0, 0), (1, 700)))
        return _append(None, shape, R, new, past, G, axes, rot, adjacent, page, major, sizes)
    if op == "decode":
        most = MOST[op] / (2 * Hkv * Dh * e)
        R = _log(rng, 1, 256)
        hi = _log(rng, 1, max(2, min(131072, most / R)))
        return _decode(None, shape, R, (max(1, hi // rng.choice((1, 1, 8, 64))), hi), page, major, sizes)
    if op == "prune":
        G = rng.choice((1, 2, 4))
        keep = rng.choice(((1, 9), (1, 8), (1, 16), (3, 8)))
        most = MOST[op] / (4 * G * Hkv * Dh * e)
        R = _log(rng, 1, 64)
        hi = _log(rng, 8, max(9, min(16384, (most / R - 70) * keep[1] / keep[0])))
        return _prune(None, shape, R, G, (max(4, hi // rng.choice((1, 4))), hi), (2, 128), keep, page, major, sizes)
    G = rng.choice((1, 2, 4))
    return _copy(None, shape, _log(rng, 1, min(65536, MOST[op] / (4 * G * Hkv * Dh * e * page))), G, page, major)


# ------------------------------------------------------------------- sizes
def _lengths(c):
    """Tokens per sequence: new ones (append), all (decode), visual ones (prune)."""
    r = random.Random(c["sizes"])
    return [min(c["hi"], max(c["lo"], _log(r, c["lo"], c["hi"]))) for _ in range(c["R"])]


def _past(c):
    r = random.Random(c["sizes"] + 1)
    return [r.randint(c["past_lo"], c["past_hi"]) for _ in range(c["R"])]


def _prune_sizes(c):
    """Visual tokens, kept ones, the visual span's start and the whole length of each sequence."""
    r = random.Random(c["sizes"] + 2)
    N = _lengths(c)
    K = [-(-n * c["keep_num"] // c["keep_den"]) for n in N]
    text = [r.randint(c["text_lo"], c["text_hi"]) for _ in N]
    return N, K, [t // 4 for t in text], [n + t for n, t in zip(N, text)]


def _cu(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def _up(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    Hq, Hkv, Dh = c["Hq"], c["Hkv"], c["Dh"]
    if c["op"] == "rotary":
        n = c["G"] * c["T"] * (Hq + Hkv)
        return {"bytes": 2 * n * Dh * e + 4 * c["axes"] * c["T"], "flops": 3 * n * c["rot"]}
    if c["op"] == "append":
        T = sum(_lengths(c))
        return {"bytes": 2 * c["G"] * T * (Hq + 2 * Hkv) * Dh * e + 4 * c["axes"] * T, "flops": 3 * c["G"] * T * (Hq + Hkv) * c["rot"]}
    if c["op"] == "decode":
        L = sum(_lengths(c))
        return {"bytes": 2 * L * Hkv * Dh * e + 2 * c["R"] * Hq * Dh * e + 4 * c["R"] * Hq + 4 * (L // c["page"]), "flops": 4 * L * Hq * Dh}
    if c["op"] == "prune":
        N, K, _, P = _prune_sizes(c)
        rows = sum(p - n + k for n, k, p in zip(N, K, P))
        return {"bytes": 4 * c["G"] * rows * Hkv * Dh * e + 4 * sum(K), "flops": 0}
    return {"bytes": 4 * c["G"] * c["n"] * c["page"] * Hkv * Dh * e + 8 * c["n"], "flops": 0}


# ------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _pool(gen, c, pages, dtype):
    shape = (c["G"], pages, c["page"], c["Hkv"], c["Dh"]) if c["token_major"] else (c["G"], pages, c["Hkv"], c["page"], c["Dh"])
    out = torch.empty(shape, device="cuda", dtype=dtype)
    for layer in out:  # a layer at a time: the draw in 32 bits is large
        layer.copy_(torch.randn(layer.shape, generator=gen, device="cuda", dtype=torch.float32))
    return out


def _view(pool, c):
    """The pool as [G][pages][Hkv][page][Dh], whatever lies where."""
    return pool.transpose(2, 3) if c["token_major"] else pool


def _table(ids, need):
    """Page table rows taken one after the other from `ids`; entries behind a sequence's last page are 0."""
    t = np.zeros((len(need), max(1, max(need))), np.int32)
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = ids[at:at + n]
        at += n
    return t


def _positions(c, T, starts, lengths, rng):
    """Positions of a prompt's tokens: their index on one axis, or frames of 16 x 16 patches in time, height and width."""
    at = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, lengths)]) if len(starts) else np.zeros(0, np.int64)
    at = at[:T] + c.get("far", 0)
    if c["axes"] == 1:
        return at[None]
    jitter = rng.integers(0, 3)
    return np.stack([at // 256 + jitter, (at // 16) % 16 + at // 256, at % 16 + at // 256])


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dtype = DTYPES[c["dtype"]]
    Hq, Hkv, Dh = c["Hq"], c["Hkv"], c["Dh"]
    s = {"case": c}
    if c["op"] in ("rotary", "append"):
        F = c["rot"] // 2
        s["inv_freq"] = torch.from_numpy((10000.0 ** (-np.arange(F) / F)).astype(np.float32)).cuda()
        # one axis, or a quarter of the frequencies in time and the rest in height and width
        split = [F] if c["axes"] == 1 else [F // 4, (F - F // 4) // 2, F - F // 4 - (F - F // 4) // 2]
        s["axis_h"] = np.repeat(np.arange(c["axes"]), split).astype(np.int32)
        s["axis"] = _up(s["axis_h"])
    if c["op"] == "rotary":
        T = c["T"]
        n = -(-T // 16512)
        s["pos"] = _up(_positions(c, T, [0] * n, [16512] * n, rng))
        s["q"] = _normal(gen, (c["G"], T, Hq, Dh), dtype)
        s["k"] = _normal(gen, (c["G"], T, Hkv, Dh), dtype)
    elif c["op"] == "append":
        new, past = _lengths(c), _past(c)
        T = sum(new)
        s["cu_h"] = _cu(new)
        s["cu"] = _up(s["cu_h"])
        s["lens_h"] = np.asarray([a + b for a, b in zip(new, past)], np.int32)
        need = [-(-int(n) // c["page"]) for n in s["lens_h"]]
        s["table_h"] = _table(rng.permutation(sum(need)), need)
        s["pos"] = _up(_positions(c, T, past, new, rng))
        s["q"] = _normal(gen, (c["G"], T, Hq, Dh), dtype)
        s["k"] = _normal(gen, (c["G"], T, Hkv, Dh), dtype)
        s["v"] = _normal(gen, (c["G"], T, Hkv, Dh), dtype)
        s["k_pool"], s["v_pool"] = _pool(gen, c, sum(need), dtype), _pool(gen, c, sum(need), dtype)
    elif c["op"] == "decode":
        s["lens_h"] = np.asarray(_lengths(c), np.int32)
        need = [-(-int(n) // c["page"]) for n in s["lens_h"]]
        s["table_h"] = _table(rng.permutation(sum(need)), need)
        s["q"] = _normal(gen, (c["R"], Hq, Dh), dtype)
        s["k_pool"], s["v_pool"] = _pool(gen, c, sum(need), dtype), _pool(gen, c, sum(need), dtype)
    elif c["op"] == "prune":
        N, K, vis, P = _prune_sizes(c)
        M = [p - n + k for p, n, k in zip(P, N, K)]
        s["lens_h"], s["after_h"] = np.asarray(P, np.int32), np.asarray(M, np.int32)
        need, later = [-(-p // c["page"]) for p in P], [-(-m // c["page"]) for m in M]
        ids = rng.permutation(sum(need) + sum(later))
        s["table_h"], s["into_h"] = _table(ids, need), _table(ids[sum(need):], later)
        s["into"] = _up(s["into_h"])
        s["vis_h"], s["cu_vis_h"], s["cu_keep_h"] = np.asarray(vis, np.int32), _cu(N), _cu(K)
        s["vis"], s["cu_vis"], s["cu_keep"] = _up(s["vis_h"]), _up(s["cu_vis_h"]), _up(s["cu_keep_h"])
        s["kept"] = _up(np.concatenate([np.sort(rng.choice(n, k, replace=False)) for n, k in zip(N, K)]))
        s["after"] = torch.zeros(c["R"], dtype=torch.int32, device="cuda")
        s["k_pool"], s["v_pool"] = _pool(gen, c, len(ids), dtype), _pool(gen, c, len(ids), dtype)
    else:
        ids = rng.permutation(2 * c["n"]).astype(np.int32)
        s["src_h"], s["dst_h"] = ids[:c["n"]].copy(), ids[c["n"]:].copy()
        s["src"], s["dst"] = _up(s["src_h"]), _up(s["dst_h"])
        s["k_pool"], s["v_pool"] = _pool(gen, c, 2 * c["n"], dtype), _pool(gen, c, 2 * c["n"], dtype)
    if "table_h" in s:
        s["table"], s["lens"] = _up(s["table_h"]), _up(s["lens_h"])
    if own:
        _handles(s)
    return s


def _handles(s):
    """The library's views of the tensors above, which a program makes once and keeps."""
    from paper_2607_27952_amd import last
    c = s["case"]
    if "axis_h" in s:
        s["rot"] = last.Rotary(inv_freq=s["inv_freq"], axis=s["axis"], axis_h=s["axis_h"], n_axes=c["axes"], adjacent=c["adjacent"])
    if "k_pool" in s:
        s["cache"] = last.Cache(_view(s["k_pool"], c), _view(s["v_pool"], c))
    if "table_h" in s:
        s["pages"] = last.Pages(table_h=s["table_h"], lens_h=s["lens_h"], table=s["table"], lens=s["lens"])
    if c["op"] == "decode":
        s["ws"] = last.decode_attention_workspace(s["cache"], s["pages"], c["Hq"])
        s["ws"] = torch.empty(max(256, s["ws"]), dtype=torch.uint8, device="cuda")
    if c["op"] == "prune":
        s["pruned"] = last.Pages(table_h=s["into_h"], lens_h=s["after_h"], table=s["into"], lens=s["after"])


# --------------------------------------------------------------- the calls
def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    return {"rotary": _plain_rotary, "append": _plain_append, "decode": _plain_decode, "prune": _plain_prune, "copy": _plain_copy}[c["op"]](s, c)


def _own(s, c):
    from paper_2607_27952_amd import last
    if c["op"] == "rotary":
        q, k = last.rotary(s["rot"], s["pos"], s["q"], s["k"], inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["op"] == "append":
        q = last.rotary_append(s["rot"], s["cache"], s["pages"], s["pos"], s["q"], s["k"], s["v"], cu_new_h=s["cu_h"], cu_new=s["cu"])
        return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if c["op"] == "decode":
        out, lse = last.decode_attention(s["cache"], s["pages"], s["q"], want_lse=True, ws=s["ws"])
        return {"out": out, "lse": lse}
    if c["op"] == "prune":
        last.cache_prune(s["cache"], s["pages"], s["pruned"], s["vis_h"], s["cu_vis_h"], s["kept"], s["cu_keep_h"], vis_start=s["vis"],
                         cu_vis=s["cu_vis"], cu_keep=s["cu_keep"])
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "lens": s["after"]}
    last.cache_copy(s["cache"], s["src_h"], s["dst_h"], src=s["src"], dst=s["dst"])
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}


# --------------------------------------------------------- the plain forms
def _turn(x, cos, sin, c):
    """x [G][T][heads][Dh] turned by the angles [T][F], in 32 bits, rounded once."""
    F = c["rot"] // 2
    y = x.float()
    cos, sin = cos[None, :, None], sin[None, :, None]
    out = y.clone()
    if c["adjacent"]:
        a, b = y[..., 0:2 * F:2], y[..., 1:2 * F:2]
        out[..., 0:2 * F:2] = a * cos - b * sin
        out[..., 1:2 * F:2] = b * cos + a * sin
    else:
        a, b = y[..., :F], y[..., F:2 * F]
        out[..., :F] = a * cos - b * sin
        out[..., F:2 * F] = b * cos + a * sin
    return out.to(x.dtype)


def _angles(s):
    a = s["pos"][s["axis"].long()].double().t() * s["inv_freq"].double()  # far positions need 64 bits
    return a.cos().float(), a.sin().float()


def _plain_rotary(s, c):
    cos, sin = _angles(s)
    sin = -sin if c["inverse"] else sin
    return {"q": _turn(s["q"], cos, sin, c), "k": _turn(s["k"], cos, sin, c)}


def _plain_append(s, c):
    cos, sin = _angles(s)
    T = s["q"].shape[1]
    counts = s["cu"][1:] - s["cu"][:-1]
    seq = torch.repeat_interleave(torch.arange(c["R"], device="cuda"), counts, output_size=T)
    at = (s["lens"] - s["cu"][1:])[seq].long() + torch.arange(T, device="cuda")
    page, slot = s["table"][seq, at // c["page"]].long(), at % c["page"]
    k_pool, v_pool = _view(s["k_pool"], c), _view(s["v_pool"], c)
    k_pool[:, page, :, slot] = _turn(s["k"], cos, sin, c).transpose(0, 1)
    v_pool[:, page, :, slot] = s["v"].transpose(0, 1)
    return {"q": _turn(s["q"], cos, sin, c), "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_decode(s, c):
    R, Hq, Hkv, Dh = c["R"], c["Hq"], c["Hkv"], c["Dh"]
    L = s["table"].shape[1] * c["page"]
    k = _view(s["k_pool"], c)[0][s["table"].long()].float().transpose(1, 2).reshape(R, Hkv, L, Dh)
    v = _view(s["v_pool"], c)[0][s["table"].long()].float().transpose(1, 2).reshape(R, Hkv, L, Dh)
    q = s["q"].float().reshape(R, Hkv, Hq // Hkv, Dh)
    a = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(Dh)
    a = a.masked_fill(torch.arange(L, device="cuda") >= s["lens"][:, None, None, None], -math.inf)
    m = a.amax(-1, keepdim=True)
    p = (a - m).exp()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total
    return {"out": out.reshape(R, Hq, Dh).to(s["q"].dtype), "lse": (m + total.log()).reshape(R, Hq)}


def _plain_prune(s, c):
    R, page = c["R"], c["page"]
    N, K = s["cu_vis"][1:] - s["cu_vis"][:-1], s["cu_keep"][1:] - s["cu_keep"][:-1]
    M = s["lens"] - N + K
    total = int(s["after_h"].sum())
    seq = torch.repeat_interleave(torch.arange(R, device="cuda"), M, output_size=total)
    i = torch.arange(total, device="cuda") - (M.cumsum(0) - M)[seq]
    vis, n, k = s["vis"][seq], N[seq], K[seq]
    slot = (s["cu_keep"][:-1][seq] + i - vis).clamp(0, s["kept"].numel() - 1)
    old = torch.where(i < vis, i, torch.where(i < vis + k, vis + s["kept"][slot], i - k + n)).long()
    a, b = s["table"][seq, old // page].long(), old % page
    x, y = s["into"][seq, i // page].long(), i % page
    k_pool, v_pool = _view(s["k_pool"], c), _view(s["v_pool"], c)
    k_pool[:, x, :, y] = k_pool[:, a, :, b]
    v_pool[:, x, :, y] = v_pool[:, a, :, b]
    s["after"].copy_(M)
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "lens": s["after"]}


def _plain_copy(s, c):
    src, dst = s["src"].long(), s["dst"].long()
    s["k_pool"][:, dst] = s["k_pool"][:, src]
    s["v_pool"][:, dst] = s["v_pool"][:, src]
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}


# --------------------------------------------------------- in 64 bits
def _exact_turn(x, s, c, sign):
    """Every pair of x as a complex number times exp(i angle), a slice of tokens at a time."""
    F = c["rot"] // 2
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    first, second = (slice(0, 2 * F, 2), slice(1, 2 * F, 2)) if c["adjacent"] else (slice(0, F), slice(F, 2 * F))
    for t in range(0, x.shape[1], 16384):
        part = x[:, t:t + 16384].double()
        angle = torch.stack([s["pos"][int(s["axis_h"][i]), t:t + 16384].double() * float(s["inv_freq"][i]) for i in range(F)], 1)
        z = torch.complex(part[..., first], part[..., second]) * torch.polar(torch.ones_like(angle), sign * angle)[None, :, None]
        part[..., first], part[..., second] = z.real, z.imag
        out[:, t:t + 16384] = part
    return out


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "rotary":
        sign = -1.0 if c["inverse"] else 1.0
        return {"q": _exact_turn(s["q"], s, c, sign), "k": _exact_turn(s["k"], s, c, sign)}
    if c["op"] == "decode":
        Hq, Hkv, Dh, page = c["Hq"], c["Hkv"], c["Dh"], c["page"]
        out = torch.empty((c["R"], Hq, Dh), dtype=torch.float64, device="cuda")
        lse = torch.empty((c["R"], Hq), dtype=torch.float64, device="cuda")
        for r in range(c["R"]):
            n = int(s["lens_h"][r])
            ids = torch.from_numpy(s["table_h"][r, :-(-n // page)].astype(np.int64)).cuda()
            for h in range(Hkv):
                k = _view(s["k_pool"], c)[0, ids, h].reshape(-1, Dh)[:n].double()
                v = _view(s["v_pool"], c)[0, ids, h].reshape(-1, Dh)[:n].double()
                heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
                a = s["q"][r, heads].double() @ k.t() * Dh ** -0.5
                lse[r, heads] = torch.logsumexp(a, -1)
                out[r, heads] = (a - lse[r, heads, None]).exp() @ v
        return {"out": out, "lse": lse}
    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    if c["op"] == "copy":
        for a, b in zip(s["src_h"].tolist(), s["dst_h"].tolist()):
            k_pool[:, b] = k_pool[:, a]
            v_pool[:, b] = v_pool[:, a]
        return {"k_pool": k_pool, "v_pool": v_pool}
    page = c["page"]
    k_at, v_at = _view(k_pool, c), _view(v_pool, c)
    if c["op"] == "append":
        k = _exact_turn(s["k"], s, c, 1.0)
        for r in range(c["R"]):
            a, b = int(s["cu_h"][r]), int(s["cu_h"][r + 1])
            at = np.arange(int(s["lens_h"][r]) - (b - a), int(s["lens_h"][r]))
            x, y = _up(s["table_h"][r][at // page], np.int64), _up(at % page, np.int64)
            k_at[:, x, :, y] = k[:, a:b].transpose(0, 1)
            v_at[:, x, :, y] = s["v"][:, a:b].double().transpose(0, 1)
        return {"q": _exact_turn(s["q"], s, c, 1.0), "k_pool": k_pool, "v_pool": v_pool}
    for r in range(c["R"]):
        start, N = int(s["vis_h"][r]), int(s["cu_vis_h"][r + 1] - s["cu_vis_h"][r])
        kept = s["kept"][int(s["cu_keep_h"][r]):int(s["cu_keep_h"][r + 1])].cpu().numpy()
        old = np.concatenate([np.arange(start), start + kept, np.arange(start + N, int(s["lens_h"][r]))])
        new = np.arange(len(old))
        a, b = _up(s["table_h"][r][old // page], np.int64), _up(old % page, np.int64)
        x, y = _up(s["into_h"][r][new // page], np.int64), _up(new % page, np.int64)
        k_at[:, x, :, y] = k_at[:, a, :, b]
        v_at[:, x, :, y] = v_at[:, a, :, b]
    return {"k_pool": k_pool, "v_pool": v_pool, "lens": None}
