"""Positions and the paged cache, as cases that can be timed and compared: the operators' plain forms in elementary torch
operations, and the library's calls.

  rope     rotary positions of the queries and keys of a projection, forward or backward
  append   one call that rotates q and k and writes k and v into the pages of a cache (bf16, or 4 bits with a scale per 32 elements)
  paged    one new query per head over the pages of a cache, one table of pages and one length per sequence

A page of a bf16 cache is [K/V head][K, V][key][d].  A page of a 4-bit cache holds, for each K/V head, blocks of 16 keys of 18 d
bytes: K codes (8 d bytes), K scales (d), V codes (8 d), V scales (d); `_split4` and `_join4` state the order inside them.
A code c of 0..15 stands for (c - 8) times its group's scale; a group is 32 neighbouring elements of a head.
"""
import math

import torch

own = False

F64, F32, BF16 = torch.float64, torch.float32, torch.bfloat16
DEV = "cuda" if torch.cuda.is_available() else "cpu"


# ------------------------------------------------------------------------------------------------------------------- cases

def _rope(name, T, n, H, Hk, d, d_rot, layout, factor, dtype, backward, far):
    """T tokens: sequences of n tokens that start at position 0, or (far > 0) single tokens at positions below `far`."""
    return {"name": name, "kind": "rope", "T": T, "n": n, "H": H, "Hk": Hk, "d": d, "d_rot": d_rot, "layout": layout, "factor": factor,
            "dtype": dtype, "backward": backward, "far": far}


def _append(name, fmt, seqs, tokens, past, H, Hk, d, d_rot, layout, page):
    """`tokens` tokens, of `seqs` sequences in ragged shares, each behind up to `past` tokens that are in the cache already."""
    return {"name": name, "kind": "append", "fmt": fmt, "seqs": seqs, "tokens": tokens, "past": past, "H": H, "Hk": Hk, "d": d,
            "d_rot": d_rot, "layout": layout, "page": page}


def _paged(name, fmt, B, n, ragged, H, Hk, d, page):
    """B sequences of n keys each, or (ragged) of 0 to n keys."""
    return {"name": name, "kind": "paged", "fmt": fmt, "B": B, "n": n, "ragged": ragged, "H": H, "Hk": Hk, "d": d, "page": page}


def listed():
    return [
        # a decoding step of a small batch, far into long conversations: all latency
        _rope("rope_step", 8, 1, 32, 8, 128, 128, "half", 1.0, "bf16", False, 131072),
        # the training step of two causal sequences: the gradients of rotated q and k turned back
        _rope("rope_train_bwd", 8192, 4096, 16, 16, 128, 128, "half", 1.0, "bf16", True, 0),
        # a long sequence, half of each head rotated in adjacent pairs, scaled for a longer context
        _rope("rope_long_partial", 16384, 16384, 16, 16, 128, 64, "pairs", 1.25, "bf16", False, 0),
        # full precision, a head size off the powers of two, a ragged number of tokens
        _rope("rope_f32_ragged", 3001, 3001, 8, 2, 80, 32, "half", 1.0, "f32", True, 0),
        # one token of each of 64 conversations into a 4-bit cache
        _append("append_step_int4", "int4", 64, 64, 30, 32, 8, 128, 128, "half", 16),
        # prompts of a few sequences into a bf16 cache
        _append("append_prompt_bf16", "bf16", 3, 8192, 0, 32, 8, 128, 128, "half", 64),
        # a ragged prompt into a 4-bit cache of small pages
        _append("append_prompt_int4", "int4", 2, 5000, 333, 32, 8, 128, 128, "pairs", 16),
        # one short conversation, one K/V head per query head: latency
        _paged("paged_short_bf16", "bf16", 1, 1000, False, 16, 16, 64, 16),
        # a batch over long bf16 caches with grouped heads: 1.07 GB read
        _paged("paged_long_bf16", "bf16", 8, 32768, False, 32, 8, 128, 64),
        # one conversation over a 4-bit cache: latency
        _paged("paged_short_int4", "int4", 1, 5000, False, 32, 8, 128, 16),
        # a served batch of 64 conversations of all lengths over 4-bit pages
        _paged("paged_batch_int4", "int4", 64, 8192, True, 32, 8, 128, 32),
        # a batch over very long 4-bit caches: 1.21 GB read
        _paged("paged_long_int4", "int4", 8, 131072, False, 32, 8, 128, 64),
    ]


_MOST_ROPE, _MOST_APPEND, _MOST_CACHE = 2.7e8, 1.8e8, 1.05e9


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, a third of each kind."""
    kind = rng.choice(("rope", "append", "paged"))
    while True:
        if kind == "rope":
            H, dtype, d = rng.choice((8, 16, 32)), rng.choice(("bf16", "bf16", "bf16", "f32")), rng.choice((64, 128, 128, 80, 96, 256))
            d_rot = rng.choice((d, d, 32, 16 * (d // 32)))
            T, far = _log(rng, 1, 16384), 0
            if T < 256 and rng.random() < 0.7:
                far = _log(rng, 256, 1 << 20)
            c = _rope("", T, 1 if far else T if rng.random() < 0.5 else max(1, T // 3), H, H // rng.choice((1, 4, 8)), d, d_rot,
                      rng.choice(("half", "half", "pairs")), rng.choice((1.0, 1.0, 1.25)), dtype, rng.random() < 0.4, far)
            fits = work(c)["bytes"] <= _MOST_ROPE
        elif kind == "append":
            H, d = rng.choice((8, 16, 32)), rng.choice((64, 128, 128))
            tokens, past = _log(rng, 1, 8192), rng.choice((0, _log(rng, 1, 512)))
            seqs = min(tokens, rng.choice((1, 3, 16, 64)))
            c = _append("", rng.choice(("bf16", "int4", "int4")), seqs, tokens, past, H, H // rng.choice((1, 4, 8)), d,
                        rng.choice((d, d, d // 2, 32)), rng.choice(("half", "half", "pairs")), rng.choice((16, 32, 64, 128)))
            fits = work(c)["bytes"] <= _MOST_APPEND
        else:
            H, d = rng.choice((8, 16, 32)), rng.choice((64, 128, 128))
            c = _paged("", rng.choice(("bf16", "int4", "int4")), _log(rng, 1, 96), _log(rng, 1, 65536), rng.random() < 0.5, H,
                       H // rng.choice((1, 4, 8)), d, rng.choice((16, 32, 64, 128)))
            fits = work(c)["bytes"] <= _MOST_CACHE and c["B"] * c["Hk"] * c["n"] * d <= 1.1e9
        if fits:
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------------------------ inputs

def _randn(gen, dtype, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=F32).to(dtype)


def _inv_freq(d_rot):
    return (10000.0 ** (-torch.arange(0, d_rot, 2, dtype=F64) / d_rot)).to(F32).to(DEV)


def _shares(gen, total, parts):
    """`parts` ragged shares of `total`, each at least one (host integers)."""
    cut = (torch.randperm(total - 1, generator=gen)[:parts - 1] + 1).sort().values.tolist()
    return [b - a for a, b in zip([0] + cut, cut + [total])]


def _append_plan(case, seed):
    """Host side of an append: (lengths in the cache before, new tokens, their sum) of each sequence."""
    gen = torch.Generator().manual_seed(seed)
    new = _shares(gen, case["tokens"], case["seqs"])
    past = torch.randint(0, case["past"] + 1, (case["seqs"],), generator=gen).tolist()
    return gen, new, past


def _slots_in_pool(case):
    """Keys that the pages of an append's pool hold; the same for every seed: all sequences' pages at their longest, and two spare ones."""
    per = lambda n: -(-n // case["page"])
    return (per(case["tokens"]) + case["seqs"] * (1 + per(case["past"])) + 2) * case["page"]


def _random_pool(gen, fmt, pages, Hk, page, d):
    """Pages filled with keys and values as a model leaves them: N(0,1), and for 4 bits codes and scales of such groups."""
    if fmt == "bf16":
        return _randn(gen, BF16, pages, Hk, 2, page, d)
    nb = page // 16
    low = torch.randint(1, 16, (pages, Hk, nb, 16 * d), generator=gen, device=DEV, dtype=torch.uint8)
    high = torch.randint(1, 16, (pages, Hk, nb, 16 * d), generator=gen, device=DEV, dtype=torch.uint8)
    low += high << 4
    scales = (0.23 + 0.12 * torch.rand((pages, Hk, nb, d), generator=gen, device=DEV)).to(BF16).view(torch.uint8)
    return torch.cat((low[..., :8 * d], scales[..., :d], low[..., 8 * d:], scales[..., d:]), -1).reshape(pages, Hk, nb * 18 * d)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "rope":
        T, H, Hk, d = (case[k] for k in ("T", "H", "Hk", "d"))
        dtype = F32 if case["dtype"] == "f32" else BF16
        # q and k as a projection leaves them, in one array, v behind them; the gradients of a backward pass likewise
        x = _randn(gen, dtype, T, H + 2 * Hk, d)
        pos = torch.randint(0, case["far"], (T,), generator=gen, device=DEV) if case["far"] else torch.arange(T, device=DEV) % case["n"]
        s.update(q=x[:, :H], k=x[:, H:H + Hk], pos=pos.to(torch.int32), inv_freq=_inv_freq(case["d_rot"]),
                 q_out=torch.empty((T, H, d), dtype=dtype, device=DEV), k_out=torch.empty((T, Hk, d), dtype=dtype, device=DEV))
        return s
    if case["kind"] == "append":
        T, H, Hk, d, page = (case[k] for k in ("tokens", "H", "Hk", "d", "page"))
        host, new, past = _append_plan(case, seed)
        total = _slots_in_pool(case)
        free, slot, pos = torch.randperm(total // page, generator=host).tolist(), [], []
        for n, p in zip(new, past):
            at = torch.arange(p, p + n)
            first = p // page
            mine = torch.tensor([free.pop() for _ in range((p + n - 1) // page - first + 1)])
            slot.append(mine[at // page - first] * page + at % page)
            pos.append(at)
        slot = torch.cat(slot)
        if T >= 8:
            slot[torch.randperm(T, generator=host)[:T // 8]] = -1        # padding of the batch: nothing is written for it
        x = _randn(gen, BF16, T, H + 2 * Hk, d)
        s.update(q=x[:, :H], k=x[:, H:H + Hk], v=x[:, H + Hk:], pos=torch.cat(pos).to(torch.int32).to(DEV), slot=slot.to(DEV),
                 inv_freq=_inv_freq(case["d_rot"]), q_out=torch.empty((T, H, d), dtype=BF16, device=DEV),
                 pool=_random_pool(gen, case["fmt"], total // page, Hk, page, d), every=torch.arange(total, device=DEV))
        return s
    B, n, H, Hk, d, page = (case[k] for k in ("B", "n", "H", "Hk", "d", "page"))
    width = -(-n // page)
    lens = torch.full((B,), n, device=DEV)
    if case["ragged"]:
        lens = torch.randint(0, n + 1, (B,), generator=gen, device=DEV)
        lens[0] = n
    table = torch.randperm(B * width, generator=gen, device=DEV).view(B, width).to(torch.int32)
    s.update(q=_randn(gen, BF16, B, H, d), pool=_random_pool(gen, case["fmt"], B * width, Hk, page, d), table=table, lens=lens.to(torch.int32),
             out=torch.empty((B, H, d), dtype=BF16, device=DEV), lse=torch.empty((B, H), dtype=F32, device=DEV))
    return s


# ------------------------------------------------------------------------------------------------------------- plain forms

def _turn(x, pos, inv_freq, layout, factor, backward, dtype):
    """Rotated x [T, heads, d] in `dtype`; the angles in 64 bits."""
    r = 2 * inv_freq.numel()
    angle = pos.to(F64)[:, None] * inv_freq.to(F64)[None, :]
    c, s = (factor * angle.cos()).to(dtype)[:, None, :], (factor * angle.sin()).to(dtype)[:, None, :]
    s = -s if backward else s
    x = x.to(dtype)
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    return torch.cat((turned, x[..., r:]), -1)


def _to_bf16(x):
    """64 bits to bf16 in one rounding (by way of 32 bits it would be two): half to even on the 45 bits that go."""
    bits = x.view(torch.int64)
    bits = (bits + ((1 << 44) - 1) + ((bits >> 45) & 1)) & ~((1 << 45) - 1)
    return bits.view(F64).to(BF16)


def _split4(pool, d):
    """Codes (0..15) and scales of a 4-bit pool [pages, Hk, bytes] as [pages, Hk, keys, d] and [pages, Hk, keys, d / 32]: K, then V."""
    P, Hk, size = pool.shape
    nb, g = size // (18 * d), d // 32
    rec = pool.view(P, Hk, nb, 18 * d)
    nibbles = lambda b: torch.stack((b & 15, b >> 4), -1).flatten(-2)
    scales = lambda b: b.contiguous().view(BF16)
    kc, ks, vc, vs = rec[..., :8 * d], rec[..., 8 * d:9 * d], rec[..., 9 * d:17 * d], rec[..., 17 * d:]
    # K: key, eight elements' place in the group, group, odd or even element, pair
    kc = nibbles(kc).view(P, Hk, nb, 16, 4, g, 2, 4).permute(0, 1, 2, 3, 5, 4, 7, 6).reshape(P, Hk, nb * 16, d)
    ks = scales(ks).view(P, Hk, nb, 8, 2, g).transpose(3, 4).reshape(P, Hk, nb * 16, g)
    # V: key / 8, elements / 4 of a group, key / 2 % 4, key % 2, group / 2, group % 2, element % 4
    vc = nibbles(vc).view(P, Hk, nb, 2, 8, 4, 2, g // 2, 2, 4).permute(0, 1, 2, 3, 5, 6, 7, 8, 4, 9).reshape(P, Hk, nb * 16, d)
    vs = scales(vs).view(P, Hk, nb, 4, g, 2, 2).permute(0, 1, 2, 5, 3, 6, 4).reshape(P, Hk, nb * 16, g)
    return kc, ks, vc, vs


def _join4(kc, ks, vc, vs):
    """The inverse of _split4."""
    P, Hk, page, d = kc.shape
    nb, g = page // 16, d // 32
    octets = lambda c: c[..., 0::2] | (c[..., 1::2] << 4)
    raw = lambda s: s.contiguous().view(torch.uint8)
    kc = octets(kc.view(P, Hk, nb, 16, g, 4, 4, 2).permute(0, 1, 2, 3, 5, 4, 7, 6).reshape(P, Hk, nb, 16 * d))
    ks = raw(ks.view(P, Hk, nb, 2, 8, g).transpose(3, 4).reshape(P, Hk, nb, 16 * g))
    vc = octets(vc.view(P, Hk, nb, 2, 4, 2, g // 2, 2, 8, 4).permute(0, 1, 2, 3, 8, 4, 5, 6, 7, 9).reshape(P, Hk, nb, 16 * d))
    vs = raw(vs.view(P, Hk, nb, 2, 4, 2, g).permute(0, 1, 2, 4, 6, 3, 5).reshape(P, Hk, nb, 16 * g))
    return torch.cat((kc, ks, vc, vs), -1).view(P, Hk, nb * 18 * d)


def _value4(codes, scales):
    return (codes.to(F32) - 8).unflatten(-1, (-1, 32)).mul(scales.to(F32)[..., None]).flatten(-2)


def _quantise(x):
    """bf16 [..., d] to codes and scales: the largest of 32 at 7, halves to even."""
    x = x.to(F32).unflatten(-1, (-1, 32))
    most = x.abs().amax(-1)
    scale = (most / 7).to(BF16)
    scale = torch.where(most < 2.0 ** -100, torch.zeros_like(scale), scale)
    step = scale.to(F32)[..., None]
    codes = torch.where(step > 0, (x / step).round().clamp(-7, 7), torch.zeros_like(x)) + 8
    return codes.flatten(-2).to(torch.uint8), scale


def _put(rows, slot, new):
    """`new` [T, Hk, ...] at the keys `slot` of rows [pages, Hk, page, ...]; a negative slot writes nothing."""
    P, Hk, page = rows.shape[:3]
    keys = rows.transpose(1, 2).reshape(P * page, Hk, -1)
    keys = torch.cat((keys, keys[:1]))                     # one key more, for what is not written
    keys[torch.where(slot < 0, torch.full_like(slot, P * page), slot)] = new.reshape(new.shape[0], Hk, -1)
    return keys[:P * page].view(P, page, Hk, -1).transpose(1, 2).contiguous()


def _by_token(rows):
    """[pages, Hk, page, d] as [keys, Hk, d]."""
    return rows.transpose(1, 2).flatten(0, 1)


def _plain_rope(s, c):
    turn = lambda x: _turn(x, s["pos"], s["inv_freq"], c["layout"], c["factor"], c["backward"], F32).to(x.dtype)
    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _plain_append(s, c):
    q = _turn(s["q"], s["pos"], s["inv_freq"], c["layout"], 1.0, False, F32).to(BF16)
    # the border between two bf16 values, and between two codes, needs more than 32 bits
    k = _to_bf16(_turn(s["k"], s["pos"], s["inv_freq"], c["layout"], 1.0, False, F64))
    if c["fmt"] == "bf16":
        s["pool"][:, :, 0] = _put(s["pool"][:, :, 0], s["slot"], k)
        s["pool"][:, :, 1] = _put(s["pool"][:, :, 1], s["slot"], s["v"])
        return {"q": q, "pool": s["pool"]}
    new = (*_quantise(k), *_quantise(s["v"]))
    parts = [_put(rows, s["slot"], x) for rows, x in zip(_split4(s["pool"], c["d"]), new)]
    s["pool"].copy_(_join4(*parts))
    return {"q": q, "k": _by_token(_value4(parts[0], parts[1])).to(BF16), "v": _by_token(_value4(parts[2], parts[3])).to(BF16)}


def _plain_paged(s, c):
    B, H, Hk, d = c["B"], c["H"], c["Hk"], c["d"]
    if c["fmt"] == "bf16":
        keys, values = s["pool"][:, :, 0].to(F32), s["pool"][:, :, 1].to(F32)
    else:
        kc, ks, vc, vs = _split4(s["pool"], d)
        keys, values = _value4(kc, ks), _value4(vc, vs)
    table = s["table"].long()
    keys = keys[table].transpose(1, 2).flatten(2, 3)       # [B, Hk, width * page, d]
    values = values[table].transpose(1, 2).flatten(2, 3)
    there = torch.arange(keys.shape[2], device=keys.device)[None, :] < s["lens"][:, None]
    q = s["q"].to(F32).view(B, Hk, H // Hk, d)
    score = (q @ keys.transpose(-1, -2)) * d ** -0.5
    score = score.masked_fill(~there[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    p = (score - torch.where(most.isinf(), torch.zeros_like(most), most)).exp()
    total = p.sum(-1, keepdim=True)
    out = (p @ values.masked_fill(~there[:, None, :, None], 0)) / torch.where(total > 0, total, torch.ones_like(total))
    return {"out": out.reshape(B, H, d).to(BF16), "lse": (most + total.log()).view(B, H)}


# --------------------------------------------------------------------------------------------------------- the library's calls

def _plan(s, make):
    """The descriptors (and workspace) that a program makes once and keeps beside its buffers."""
    if "plan" not in s:
        s["plan"] = make()
    return s["plan"]


def _layout(mb, name):
    return mb.MOA_ROPE_HALF if name == "half" else mb.MOA_ROPE_PAIRS


def _cache(mb, c, pages):
    return mb.make_cache_desc(pages, c["page"], c["Hk"], c["d"], mb.MOA_CACHE_BF16 if c["fmt"] == "bf16" else mb.MOA_CACHE_INT4)


def _own_rope(mb, s, c):
    desc = _plan(s, lambda: mb.make_rope_desc(c["T"], c["H"], c["Hk"], c["d"], c["d_rot"], _layout(mb, c["layout"]), c["factor"],
                                              mb.MOA_F32 if c["dtype"] == "f32" else mb.MOA_BF16, q_stride=s["q"].stride()[:2],
                                              k_stride=s["k"].stride()[:2]))
    (mb.moa_rope_bwd if c["backward"] else mb.moa_rope_fwd)(desc, s["pos"], s["inv_freq"], s["q"], s["k"], s["q_out"], s["k_out"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(mb, s, c):
    def make():
        cache = _cache(mb, c, s["pool"].shape[0])
        total = s["every"].numel()
        desc = mb.make_append_desc(cache, c["tokens"], c["H"], c["d_rot"], _layout(mb, c["layout"]), q_stride=s["q"].stride()[:2],
                                   k_stride=s["k"].stride()[:2], v_stride=s["v"].stride()[:2])
        values = [torch.empty((total, c["Hk"], c["d"]), dtype=BF16, device=DEV) for _ in range(2)] if c["fmt"] == "int4" else None
        return desc, mb.make_gather_desc(cache, total), values

    desc, gather, values = _plan(s, make)
    mb.moa_kv_append(desc, s["q"], s["k"], s["v"], s["pos"], s["slot"], s["inv_freq"], s["q_out"], s["pool"])
    if values is None:
        return {"q": s["q_out"], "pool": s["pool"]}
    mb.moa_kv_gather(gather, s["pool"], s["every"], *values)           # the values that the cache now stands for
    return {"q": s["q_out"], "k": values[0], "v": values[1]}


def _own_paged(mb, s, c):
    def make():
        desc = mb.make_paged_decode_desc(_cache(mb, c, s["pool"].shape[0]), c["B"], c["H"], s["table"].shape[1], c["d"] ** -0.5)
        return desc, torch.empty(max(16, mb.moa_paged_decode_workspace_bytes(desc)), dtype=torch.uint8, device=DEV)

    desc, ws = _plan(s, make)
    mb.moa_paged_decode(desc, s["q"], s["pool"], s["table"], s["lens"], s["out"], s["lse"], ws)
    return {"out": s["out"], "lse": s["lse"]}


def run(s):
    c = s["case"]
    if own:
        from paper_2609_33916_b200 import binding as mb
        return {"rope": _own_rope, "append": _own_append, "paged": _own_paged}[c["kind"]](mb, s, c)
    return {"rope": _plain_rope, "append": _plain_append, "paged": _plain_paged}[c["kind"]](s, c)


# ----------------------------------------------------------------------------------------------------------------- work

def work(case):
    """Every input read once and every output written once (a 4-bit append also reads its pool back as bf16)."""
    d, H, Hk = case["d"], case["H"], case["Hk"]
    if case["kind"] == "rope":
        size, T = (4 if case["dtype"] == "f32" else 2), case["T"]
        return {"bytes": T * (2.0 * (H + Hk) * d * size + 4) + 2.0 * case["d_rot"], "flops": 3.0 * T * (H + Hk) * case["d_rot"]}
    per_key = 2 * d * 2 if case["fmt"] == "bf16" else d * 9 / 8
    if case["kind"] == "append":
        T, total = case["tokens"], _slots_in_pool(case)
        written = 7 * T / 8 if T >= 8 else T
        back = 0 if case["fmt"] == "bf16" else total * Hk * (per_key + 4.0 * d) + 8 * total
        return {"bytes": T * (2.0 * H * d * 2 + Hk * 4.0 * d + 12) + written * Hk * per_key + back,
                "flops": 3.0 * T * (H + Hk) * case["d_rot"]}
    keys = case["B"] * case["n"] * (0.5 if case["ragged"] else 1.0)
    return {"bytes": keys * Hk * per_key + case["B"] * (H * (4.0 * d + 4) + 4 + 4 * -(-case["n"] // case["page"])),
            "flops": 4.0 * keys * H * d}


# ---------------------------------------------------------------------------------------------------------------- in 64 bits

def _exact_turn(x, pos, inv_freq, layout, factor, backward):
    """The rotation as a product of complex numbers."""
    r = 2 * inv_freq.numel()
    turn = torch.polar(torch.full_like(inv_freq, factor, dtype=F64), torch.zeros_like(inv_freq, dtype=F64))
    angle = pos.double().unsqueeze(1) * inv_freq.double()
    turn = turn * torch.complex(angle.cos(), -angle.sin() if backward else angle.sin())
    y = x.double().clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., first], y[..., second]) * turn.unsqueeze(1)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _round_bits(x, bits):
    """x to `bits` significant bits, halves to even."""
    m, e = torch.frexp(x)
    return torch.ldexp((m * 2.0 ** bits).round(), e - bits)


def _exact_values4(block, d, values):
    """Keys or values of 4-bit blocks [..., 9 d bytes] as [..., 16, d], element by element from the places of codes and scales."""
    g = d // 32
    r, x = torch.meshgrid(torch.arange(16), torch.arange(d), indexing="ij")
    grp, y = x // 32, x % 32
    if values:
        word = (r // 8) * 128 * g + ((y // 4) * 4 + (r % 8) // 2) * g * 4 + (r % 2) * g * 2 + (grp // 2) * 4
        nib = (grp % 2) * 4 + y % 4
        scale = ((r % 8) // 2) * 8 * g + grp * 8 + (r // 8) * 4 + (r % 2) * 2
    else:
        word = r * (d // 2) + ((y // 8) * g + grp) * 4
        nib = (y % 2) * 4 + (y % 8) // 2
        scale = ((r % 8) * 2 + r // 8) * 2 * g + grp * 2
    word, nib, scale = (t.to(block.device) for t in (word + nib // 2, nib, scale + 8 * d))
    code = (block[..., word].to(torch.int32) >> (4 * (nib % 2))) & 15
    bits = block[..., scale].to(torch.int32) + (block[..., scale + 1].to(torch.int32) << 8)
    return (code.double() - 8) * (bits << 16).view(F32).double()


def _exact_quantised(x):
    """What 4 bits make of x [..., d] (64 bits): the nearest of 15 multiples of the group's scale."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    scale = _round_bits(y.abs().max(-1, keepdim=True).values / 7, 8)
    return torch.where(scale > 0, (y / scale).round() * scale, 0).reshape(x.shape)


def _exact_append(case, s):
    q = _exact_turn(s["q"], s["pos"], s["inv_freq"], case["layout"], 1.0, False)
    k = _round_bits(_exact_turn(s["k"], s["pos"], s["inv_freq"], case["layout"], 1.0, False), 8)
    v = s["v"].double()
    d, page, Hk, P = case["d"], case["page"], case["Hk"], s["pool"].shape[0]
    live = (s["slot"] >= 0).nonzero().flatten()
    at = s["slot"][live]
    if case["fmt"] == "bf16":
        pool = s["pool"].double()
        pool[at // page, :, 0, at % page], pool[at // page, :, 1, at % page] = k[live], v[live]
        return {"q": q, "pool": pool}
    both = []
    for values, new in ((False, k), (True, v)):
        block = s["pool"].view(P, Hk, page // 16, 2, 9 * d)[:, :, :, int(values)]
        rows = _exact_values4(block, d, values).reshape(P, Hk, page, d).permute(0, 2, 1, 3).reshape(P * page, Hk, d)
        rows[at] = _exact_quantised(new[live])
        both.append(rows)
    return {"q": q, "k": both[0], "v": both[1]}


def _exact_paged(case, s):
    B, H, Hk, d, page = (case[k] for k in ("B", "H", "Hk", "d", "page"))
    out, lse = torch.zeros((B, H, d), dtype=F64, device=DEV), torch.full((B, H), -math.inf, dtype=F64, device=DEV)
    lens = s["lens"].tolist()
    for b in range(B):
        if lens[b] == 0:
            continue
        pages = s["pool"][s["table"][b, :-(-lens[b] // page)].long()]
        for h in range(Hk):
            if case["fmt"] == "bf16":
                key, value = pages[:, h, 0].double(), pages[:, h, 1].double()
            else:
                blocks = pages[:, h].reshape(-1, 2, 9 * d)
                key, value = _exact_values4(blocks[:, 0], d, False), _exact_values4(blocks[:, 1], d, True)
            key, value = key.reshape(-1, d)[:lens[b]], value.reshape(-1, d)[:lens[b]]
            heads = slice(h * (H // Hk), (h + 1) * (H // Hk))
            score = (s["q"][b, heads].double() @ key.T) / math.sqrt(d)
            lse[b, heads] = score.logsumexp(-1)
            out[b, heads] = score.softmax(-1) @ value
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        turn = lambda x: _exact_turn(x, s["pos"], s["inv_freq"], case["layout"], case["factor"], case["backward"])
        return {"q": turn(s["q"]), "k": turn(s["k"])}
    return _exact_append(case, s) if case["kind"] == "append" else _exact_paged(case, s)
