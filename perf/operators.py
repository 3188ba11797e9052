"""Cases of the operators around attention that stand beside the linear layer and the plain attention of the library.

Four families, each with its own ranges (see draw):
  rope     rotary positions with several axes on the queries and keys of packed tokens, with or without the norm of every head
  packed   attention inside each of several sequences laid end to end, grouped heads, causal or not
  store    keys and values of new tokens into a cache of 8-bit pages, and the values that the pages written to then hold
  cached   attention of new tokens (one, or a frame of them) over such a cache

Queries and keys have unit deviation, as behind the norm of every head; so have values.  Lengths are texts ("77+4096"), so that a
case says them itself.  A cache page holds 64 tokens of one head: keys as [64][head_dim] bytes, values as [head_dim][64] bytes whose
place 16 g + 4 m + i belongs to token 16 m + 4 g + i, both e4m3, with one power-of-two scale each."""
from __future__ import annotations

import math

import torch

own = False             # False: the plain forms; True: the library's operators

PAGE = 64
EPS = 1e-6


def listed():
    return [
        # the next token of each of eight sequences, three axes, frequencies shared by the axes: the smallest call
        {"name": "rope_next_tokens", "family": "rope", "dtype": "bf16", "tokens": 8, "heads": 32, "kv_heads": 8, "head_dim": 128,
         "dims": "32+48+48", "pairing": "halves", "spectrum": "joint", "norm": False, "far": 100000},
        # a 512 x 512 picture in single precision (two axes, heads of 72, of which 8 features are not rotated)
        {"name": "rope_picture_f32", "family": "rope", "dtype": "f32", "tokens": 1024, "heads": 16, "kv_heads": 16, "head_dim": 72,
         "dims": "32+32", "pairing": "adjacent", "spectrum": "per_axis", "norm": True, "far": 64},
        # a 480p clip behind its text (time, height, width), with the norm of every head: the largest
        {"name": "rope_clip", "family": "rope", "dtype": "bf16", "tokens": 27286, "heads": 24, "kv_heads": 24, "head_dim": 128,
         "dims": "16+56+56", "pairing": "adjacent", "spectrum": "per_axis", "norm": True, "far": 64},
        # sixteen thumbnails of all shapes in one batch (heads of 72)
        {"name": "packed_thumbnails", "family": "packed", "dtype": "bf16", "lens": "64+256+196+77+15+300+144+256+400+121+1+240+90+256+330+169",
         "heads": 16, "kv_heads": 16, "head_dim": 72, "causal": False},
        # prompts of all lengths through a text encoder (causal, four query heads per key head)
        {"name": "packed_prompts", "family": "packed", "dtype": "bf16", "lens": "37+4096+512+1201+77+2048+300+3001+19+650+1500+128",
         "heads": 32, "kv_heads": 8, "head_dim": 128, "causal": True},
        # pictures of 1024 x 1024 and below with their texts: the largest
        {"name": "packed_pictures", "family": "packed", "dtype": "bf16", "lens": "4608+2381+4608+1101+589", "heads": 24, "kv_heads": 24,
         "head_dim": 128, "causal": False},
        # a reference run in single precision
        {"name": "packed_f32", "family": "packed", "dtype": "f32", "lens": "1024+77+777+256", "heads": 6, "kv_heads": 6, "head_dim": 64, "causal": False},
        # one new token for each of 16 sequences, somewhere in a page
        {"name": "store_next_tokens", "family": "store", "dtype": "bf16", "lens": "+".join(["1"] * 16), "past": "130+0+63+64+700+5+127+1000+31+77+256+511+90+12+333+640",
         "heads": 8, "head_dim": 128},
        # a frame of a 480p clip, one of a smaller clip and a text, behind what is there
        {"name": "store_frames", "family": "store", "dtype": "bf16", "lens": "1590+845+77", "past": "25440+3380+0", "heads": 24, "head_dim": 128},
        # one token of each of four short sequences: latency
        {"name": "cached_short", "family": "cached", "dtype": "bf16", "new": "1+1+1+1", "lens": "77+513+1+1200", "heads": 32, "kv_heads": 8, "head_dim": 128, "causal": True},
        # one token of each of eight sequences of up to 64 k tokens: the memory's rate
        {"name": "cached_long", "family": "cached", "dtype": "bf16", "new": "1+1+1+1+1+1+1+1", "lens": "65000+1333+30001+9000+48000+257+20000+39999",
         "heads": 32, "kv_heads": 8, "head_dim": 128, "causal": True},
        # the next frame of a 480p clip over the 16 before it and the text
        {"name": "cached_frame", "family": "cached", "dtype": "bf16", "new": "1590", "lens": "27286", "heads": 24, "kv_heads": 24, "head_dim": 128, "causal": False},
    ]


# ---- drawing cases ----------------------------------------------------------------------------------------------


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(values):
    return "+".join(str(v) for v in values)


def _numbers(text):
    return [int(v) for v in text.split("+")]


def _draw_rope(rng):
    while True:
        hd = rng.choice([64, 72, 128])
        axes = rng.choice([1, 2, 3, 3])
        rotated = hd if hd != 72 else 64
        dims = {1: [rotated], 2: [rotated // 2, rotated // 2], 3: [rotated // 4, 3 * rotated // 8, 3 * rotated // 8]}[axes]
        heads, kv_heads = rng.choice([(6, 6), (16, 16), (24, 24), (32, 8), (12, 4), (28, 4)])
        c = {"family": "rope", "dtype": rng.choice(["bf16", "bf16", "f32"]), "tokens": _log_int(rng, 1, 27286), "heads": heads, "kv_heads": kv_heads,
             "head_dim": hd, "dims": _text(dims), "pairing": rng.choice(["adjacent", "halves"]), "spectrum": rng.choice(["per_axis", "joint"]),
             "norm": rng.random() < 0.5, "far": _log_int(rng, 16, 200000)}
        if work(c)["bytes"] <= work(listed()[2])["bytes"]:
            return c


def _draw_packed(rng):
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        heads, kv_heads = rng.choice([(6, 6), (16, 16), (24, 24), (32, 8), (12, 4), (16, 2)])
        most = 6000 if dtype == "bf16" else 1500
        c = {"family": "packed", "dtype": dtype, "lens": _text(_log_int(rng, 1, most) for _ in range(_log_int(rng, 1, 24))), "heads": heads,
             "kv_heads": kv_heads, "head_dim": rng.choice([64, 72, 128]), "causal": rng.random() < 0.5}
        if work(c)["flops"] <= (work(listed()[5])["flops"] if dtype == "bf16" else 2e10):
            return c


def _draw_store(rng):
    while True:
        n = _log_int(rng, 1, 24)
        longest = rng.choice([1, 64, 2000])
        c = {"family": "store", "dtype": rng.choice(["bf16", "bf16", "f32"]), "lens": _text(_log_int(rng, 1, longest) for _ in range(n)),
             "past": _text(rng.choice([0, _log_int(rng, 1, 4000)]) for _ in range(n)), "heads": rng.choice([2, 4, 8, 16, 24]),
             "head_dim": rng.choice([64, 72, 128])}
        if work(c)["bytes"] <= work(listed()[8])["bytes"]:
            return c


def _draw_cached(rng):
    while True:
        n = _log_int(rng, 1, 24)
        longest = rng.choice([1, 1, 16, 2000])
        new = [_log_int(rng, 1, longest) for _ in range(n)]
        heads, kv_heads = rng.choice([(16, 16), (24, 24), (32, 8), (12, 4), (16, 2), (28, 4)])
        c = {"family": "cached", "dtype": "bf16", "new": _text(new), "lens": _text(v + _log_int(rng, 1, 50000) - 1 for v in new), "heads": heads,
             "kv_heads": kv_heads, "head_dim": rng.choice([64, 72, 128]), "causal": rng.random() < 0.7}
        w = work(c)
        if w["flops"] <= work(listed()[11])["flops"] and w["bytes"] <= work(listed()[10])["bytes"]:
            return c


def draw(rng):
    """One more case, of any family."""
    return rng.choice([_draw_rope, _draw_packed, _draw_store, _draw_cached])(rng)


# ---- inputs -------------------------------------------------------------------------------------------------------


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"rope": _prepare_rope, "packed": _prepare_packed, "store": _prepare_store, "cached": _prepare_cached}[case["family"]](case, g)


def _prepare_rope(c, g):
    # one layer's output [tokens, (heads + 2 kv_heads) * head_dim], of which q and k are views, as a block has them
    hd, width = c["head_dim"], (c["heads"] + 2 * c["kv_heads"]) * c["head_dim"]
    qkv = _normal(g, (c["tokens"], width), _dtype(c))
    axes = len(_numbers(c["dims"]))
    s = {"case": c, "q": qkv[:, :c["heads"] * hd].view(-1, c["heads"], hd),
         "k": qkv[:, c["heads"] * hd:(c["heads"] + c["kv_heads"]) * hd].view(-1, c["kv_heads"], hd),
         "positions": torch.randint(0, c["far"], (c["tokens"], axes), generator=g, device="cuda", dtype=torch.int32), "q_norm": None, "k_norm": None}
    if c["norm"]:
        s["q_norm"], s["k_norm"] = ((1.0 + 0.02 * torch.randn(hd, generator=g, device="cuda")).to(_dtype(c)) for _ in range(2))
    return s


def _prepare_packed(c, g):
    lens = _numbers(c["lens"])
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    qkv = _normal(g, (sum(lens), (H + 2 * Hkv) * hd), _dtype(c))
    return {"case": c, "lens": lens, "starts": _starts(lens), "q": qkv[:, :H * hd].view(-1, H, hd), "k": qkv[:, H * hd:(H + Hkv) * hd].view(-1, Hkv, hd),
            "v": qkv[:, (H + Hkv) * hd:].view(-1, Hkv, hd)}


def _prepare_cache(held, room, heads, hd, g):
    """A cache whose pages are dealt out in no order, full of tokens of unit deviation; a row of page numbers per sequence."""
    count = [-(-n // PAGE) for n in room]
    pages = sum(count)
    table = torch.zeros((len(room), max(count)), dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    at = 0
    for s, n in enumerate(count):
        table[s, :n] = order[at:at + n]
        at += n
    # the largest of 64 x head_dim normal values lies between 3.5 and 7: scales of 2^-6, and the odd 2^-7
    scale = [torch.where(torch.rand((pages, heads), generator=g, device="cuda") < 0.1, 2.0 ** -7, 2.0 ** -6) for _ in range(2)]
    k, v = (torch.randn((pages, heads, PAGE * hd), generator=g, device="cuda") for _ in range(2))
    k, v = (torch.clamp(x / s[:, :, None], -448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) for x, s in ((k, scale[0]), (v, scale[1])))
    return {"table": table, "kc": k.view(pages, heads, PAGE, hd), "vc": v.view(pages, heads, hd, PAGE), "ks": scale[0], "vs": scale[1],
            "held": torch.tensor(held, dtype=torch.int32, device="cuda")}


def _prepare_store(c, g):
    lens, past = _numbers(c["lens"]), _numbers(c["past"])
    s = _prepare_cache(past, [a + b for a, b in zip(lens, past)], c["heads"], c["head_dim"], g)
    kv = _normal(g, (sum(lens), 2 * c["heads"] * c["head_dim"]), _dtype(c))
    kv *= 1.0 + (torch.arange(sum(lens), device="cuda")[:, None] % 5 == 0)          # every fifth token is large enough for another scale now and then
    half = c["heads"] * c["head_dim"]
    # what is read back: from the start of the page that a sequence's old tokens end in
    back = [b % PAGE for b in past]
    s.update(case=c, lens=lens, past=past, starts=_starts(lens), k=kv[:, :half].view(-1, c["heads"], c["head_dim"]), v=kv[:, half:].view(-1, c["heads"], c["head_dim"]),
             read=[a + b for a, b in zip(lens, back)], read_starts=_starts([a + b for a, b in zip(lens, back)]),
             read_from=torch.tensor([b // PAGE * PAGE for b in past], dtype=torch.int32, device="cuda"))
    return s


def _prepare_cached(c, g):
    new, lens = _numbers(c["new"]), _numbers(c["lens"])
    s = _prepare_cache(lens, lens, c["kv_heads"], c["head_dim"], g)
    s.update(case=c, new=new, lens=lens, starts=_starts(new), q=_normal(g, (sum(new), c["heads"], c["head_dim"]), torch.bfloat16))
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------


def run(state):
    return {"rope": _run_rope, "packed": _run_packed, "store": _run_store, "cached": _run_cached}[state["case"]["family"]](state)


def _run_rope(s):
    c = s["case"]
    dims = _numbers(c["dims"])
    if own:
        from paper_2509_11628_amd import binding as bd
        rope = bd.make_rope(dims, theta=10000.0, pairing=bd.ROPE_ADJACENT if c["pairing"] == "adjacent" else bd.ROPE_HALVES,
                            spectrum=bd.ROPE_PER_AXIS if c["spectrum"] == "per_axis" else bd.ROPE_JOINT)
        return bd.rope_axes(rope, s["positions"], s["q"], s["k"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
    total = sum(dims)
    pos = s["positions"].double()
    if c["spectrum"] == "per_axis":
        angle = torch.cat([pos[:, a:a + 1] * 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d) for a, d in enumerate(dims)], dim=1)
    else:
        axis = torch.repeat_interleave(torch.arange(len(dims), device="cuda"), torch.tensor([d // 2 for d in dims], device="cuda"), output_size=total // 2)
        angle = pos[:, axis] * 10000.0 ** (-torch.arange(0, total, 2, device="cuda", dtype=torch.float64) / total)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotated(x, norm):
        y = x.float()
        if norm is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * norm.float()
        if c["pairing"] == "adjacent":
            a, b = y[..., 0:total:2], y[..., 1:total:2]
            z = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
        else:
            a, b = y[..., :total // 2], y[..., total // 2:total]
            z = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
        return torch.cat([z, y[..., total:]], dim=-1).to(x.dtype)

    return rotated(s["q"], s["q_norm"]), rotated(s["k"], s["k_norm"])


def _attend(q, k, v, causal):
    """Queries [n, heads, hd] over keys and values [m, kv_heads, hd], all in 32 bits; causal: the last query sees every key."""
    n, H, hd = q.shape
    m, Hkv, _ = k.shape
    score = torch.matmul(q.transpose(0, 1).reshape(Hkv, (H // Hkv) * n, hd) * (1.0 / math.sqrt(hd)), k.permute(1, 2, 0).contiguous()).view(H, n, m)
    if causal:
        hidden = torch.arange(m, device=q.device)[None, :] > torch.arange(n, device=q.device)[:, None] + (m - n)
        score = score.masked_fill(hidden, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.matmul(p.view(Hkv, (H // Hkv) * n, m), v.transpose(0, 1).contiguous()).view(H, n, hd) / p.sum(-1)[..., None]
    return o.transpose(0, 1)


def _run_packed(s):
    c = s["case"]
    if own:
        from paper_2509_11628_amd import binding as bd
        return bd.attention_packed(s["q"], s["k"], s["v"], s["starts"], causal=c["causal"])
    q, k, v = (x.float().split(s["lens"]) for x in (s["q"], s["k"], s["v"]))
    return torch.cat([_attend(a, b, d, c["causal"]) for a, b, d in zip(q, k, v)]).to(s["q"].dtype)


def _values(b, scale):
    """Bytes of pages [n, heads, ...] as the numbers they stand for."""
    return b.view(torch.float8_e4m3fn).float() * scale[:, :, None, None]


def _by_token(v):
    """Value pages [n, heads, hd, 64] in the order of the tokens: [n, heads, 64, hd]."""
    n, h, hd, _ = v.shape
    return v.view(n, h, hd, 4, 4, 4).transpose(3, 4).reshape(n, h, hd, PAGE).transpose(2, 3)


def _by_feature(v):
    """The other way round."""
    n, h, _, hd = v.shape
    return v.transpose(2, 3).reshape(n, h, hd, 4, 4, 4).transpose(3, 4).reshape(n, h, hd, PAGE)


def _places(s, lens, starts, first):
    """Page number and place in the page of tokens first, first + 1, ... of every sequence."""
    lens, total = torch.tensor(lens, device="cuda"), sum(lens)
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens, output_size=total)
    at = torch.arange(total, device="cuda") - starts.long()[seq] + first.long()[seq]
    return s["table"][seq, at // PAGE].long(), at % PAGE


def _power(e):
    """2^e of whole numbers, in 32 bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _run_store(s):
    if own:
        from paper_2509_11628_amd import binding as bd
        cache = bd.KVCache(s["kc"], s["vc"], s["ks"], s["vs"])
        bd.kv_store(cache, s["table"], s["held"], s["k"], s["v"], s["starts"])
        k, v = bd.kv_load(cache, s["table"], s["read_from"], s["read_starts"], sum(s["read"]), s["k"].dtype)
        return {"k": k, "v": v, "k_scale": s["ks"], "v_scale": s["vs"]}
    page, place = _places(s, s["lens"], s["starts"], s["held"])
    touched, back = torch.unique(page, return_inverse=True)
    # how much of each touched page was held before: the places below the first new one
    first = torch.full((len(touched),), PAGE, device="cuda").scatter_reduce(0, back, place, "amin")
    old = (torch.arange(PAGE, device="cuda")[None, :] < first[:, None])[:, None, :, None]
    out = {}
    for name, raw, scales in (("k", s["kc"], s["ks"]), ("v", s["vc"], s["vs"])):
        held = _values(raw[touched], scales[touched])
        new = torch.zeros((len(touched), s["case"]["heads"], PAGE, s["case"]["head_dim"]), device="cuda")
        new[back, :, place] = s[name].float()
        # the smallest power of two whose 448-fold reaches the largest new value, and not below the one that the old tokens have
        top = new.abs().amax((2, 3))
        m, e = torch.frexp(top / 448.0)
        e = torch.where(top > 0, torch.clamp(torch.where(m == 0.5, e - 1, e), -100, 119), -100)
        scale = torch.maximum(_power(e), torch.where(first[:, None] > 0, scales[touched], 0.0))
        x = torch.where(old, held if name == "k" else _by_token(held), new) / scale[:, :, None, None]
        b = torch.clamp(x, -448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        raw[touched] = b if name == "k" else _by_feature(b)
        scales[touched] = scale
        page, place_read = _places(s, s["read"], s["read_starts"], s["read_from"])
        held = _values(raw[page], scales[page])
        held = held if name == "k" else _by_token(held)
        out[name] = held[torch.arange(len(page), device="cuda"), :, place_read].to(s[name].dtype)
        out[name + "_scale"] = scales
    return out


def _run_cached(s):
    c = s["case"]
    if own:
        from paper_2509_11628_amd import binding as bd
        cache = bd.KVCache(s["kc"], s["vc"], s["ks"], s["vs"])
        return bd.attention_cached(s["q"], s["starts"], cache, s["table"], s["held"], causal=c["causal"])
    out = []
    for q, n, row in zip(s["q"].float().split(s["new"]), s["lens"], s["table"]):
        page = row[:-(-n // PAGE)].long()
        k, v = _values(s["kc"][page], s["ks"][page]), _by_token(_values(s["vc"][page], s["vs"][page]))
        k, v = (x.transpose(1, 2).reshape(-1, c["kv_heads"], c["head_dim"])[:n] for x in (k, v))
        out.append(_attend(q, k, v, c["causal"]))
    return torch.cat(out).to(torch.bfloat16)


# ---- work ---------------------------------------------------------------------------------------------------------


def work(case):
    """Inputs read once, outputs written once; two operations per multiply-add of the attention's products."""
    c, esz = case, 2 if case["dtype"] == "bf16" else 4
    hd = c["head_dim"]
    if c["family"] == "rope":
        n = c["tokens"] * (c["heads"] + c["kv_heads"]) * hd
        return {"bytes": 2 * n * esz + c["tokens"] * 4 * len(_numbers(c["dims"])), "flops": 6 * n}
    lens = _numbers(c["lens"])
    if c["family"] == "packed":
        pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens)
        return {"bytes": esz * sum(lens) * hd * 2 * (c["heads"] + c["kv_heads"]), "flops": 4 * c["heads"] * hd * pairs}
    if c["family"] == "store":
        back = sum(b % PAGE for b in _numbers(c["past"]))
        return {"bytes": 2 * c["heads"] * hd * (sum(lens) * (esz + 1) + (sum(lens) + back) * (esz + 1)), "flops": 4 * sum(lens) * c["heads"] * hd}
    new = _numbers(c["new"])
    pairs = sum(a * n - (a * (a - 1) // 2 if c["causal"] else 0) for a, n in zip(new, lens))
    return {"bytes": sum(lens) * c["kv_heads"] * hd * 2 + 2 * 2 * sum(new) * c["heads"] * hd, "flops": 4 * c["heads"] * hd * pairs}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "packed": _exact_packed, "store": _exact_store, "cached": _exact_cached}[case["family"]](s)


def _exact_rope(s):
    c = s["case"]
    dims = _numbers(c["dims"])
    total, hd = sum(dims), c["head_dim"]
    rate, axis, upto = [], [], 0
    for a, d in enumerate(dims):
        for j in range(d // 2):
            rate.append(math.pow(10000.0, -2.0 * j / d) if c["spectrum"] == "per_axis" else math.pow(10000.0, -2.0 * (upto + j) / total))
            axis.append(a)
        upto += d // 2
    angle = s["positions"].to(torch.float64)[:, axis] * torch.tensor(rate, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]                     # pairs as complex numbers, turned by the angle
    at = [(2 * i, 2 * i + 1) if c["pairing"] == "adjacent" else (i, i + total // 2) for i in range(total // 2)]
    first, second = [p[0] for p in at], [p[1] for p in at]
    out = []
    for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
        y = x.to(torch.float64)
        if w is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / hd + EPS) * w.to(torch.float64)
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_softmax(q, k, v, sees):
    """One head: queries over keys, `sees` where a query may look."""
    score = (q @ k.T) / math.sqrt(q.shape[1])
    if sees is not None:
        score = torch.where(sees, score, -math.inf)
    return torch.softmax(score, dim=1) @ v


def _exact_packed(s):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    q, k, v = (s[n].to(torch.float64) for n in "qkv")
    out, at = torch.empty_like(q), 0
    for n in s["lens"]:
        sees = torch.ones((n, n), dtype=torch.bool, device="cuda").tril() if c["causal"] else None
        for h in range(c["heads"]):
            out[at:at + n, h] = _exact_softmax(q[at:at + n, h], k[at:at + n, h // group], v[at:at + n, h // group], sees)
        at += n
    return out


def _code_values():
    """The 256 numbers of e4m3: sign, four bits of exponent with bias 7, three of mantissa; all ones is no number."""
    out = []
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = math.nan if e == 15 and m == 7 else (m / 8.0) * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
        out.append(-x if b & 128 else x)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _token_places():
    """Where token t of a page stands in a row of the value page."""
    return torch.tensor([16 * (t % 16 // 4) + 4 * (t // 16) + t % 4 for t in range(PAGE)], device="cuda")


def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _nearest_code(x):
    """x rounded to e4m3, ties to the even mantissa, saturating."""
    a = x.abs().clamp(max=448.0)
    step = _two_to(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign(torch.round(a / step) * step, x)


def _exact_store(s):
    codes, order = _code_values(), _token_places()
    out = {}
    for name, raw, scales in (("k", s["kc"], s["ks"]), ("v", s["vc"], s["vs"])):
        x, scale, got, at = s[name].to(torch.float64), scales.to(torch.float64), [], 0
        for n, past, row in zip(s["lens"], s["past"], s["table"].tolist()):
            for j in range(past // PAGE, (past + n - 1) // PAGE + 1):
                lo, hi = max(past, j * PAGE), min(past + n, (j + 1) * PAGE)
                page = x[at + lo - past:at + hi - past]
                sc = _two_to(torch.ceil(torch.log2(page.abs().amax((0, 2)).clamp(min=2.0 ** -120) / 448.0)).clamp(-100, 119))
                if lo > j * PAGE:                     # tokens that were there keep a scale that is large enough for them
                    was = codes[raw[row[j]].long()] * scale[row[j]][:, None, None]
                    was = was.transpose(0, 1) if name == "k" else was[..., order].permute(2, 0, 1)
                    page = torch.cat([was[:lo - j * PAGE], page])
                    sc = torch.maximum(sc, scale[row[j]])
                scale[row[j]] = sc
                got.append(_nearest_code(page / sc[None, :, None]) * sc[None, :, None])
            at += n
        out[name], out[name + "_scale"] = torch.cat(got), scale
    return out


def _exact_cached(s):
    c = s["case"]
    codes, order = _code_values(), _token_places()
    group = c["heads"] // c["kv_heads"]
    q = s["q"].to(torch.float64)
    out, at = torch.empty_like(q), 0
    for a, n, row in zip(s["new"], s["lens"], s["table"]):
        page = row.long()[:(n + PAGE - 1) // PAGE]
        sees = None
        if c["causal"] and a > 1:
            sees = torch.arange(n, device="cuda")[None] <= torch.arange(n - a, n, device="cuda")[:, None]
        for h in range(c["kv_heads"]):
            k = (codes[s["kc"][page, h].long()] * s["ks"][page, h].double()[:, None, None]).reshape(-1, c["head_dim"])[:n]
            v = (codes[s["vc"][page, h].long()][..., order] * s["vs"][page, h].double()[:, None, None]).transpose(1, 2).reshape(-1, c["head_dim"])[:n]
            for i in range(h * group, (h + 1) * group):
                out[at:at + a, i] = _exact_softmax(q[at:at + a, i], k, v, sees)
        at += a
    return out
