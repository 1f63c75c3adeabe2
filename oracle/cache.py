"""fp64 oracle of rotary positions and of the paged cache.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain numpy, the definitions written out:

    rope     angle = pos * inv_freq[i];  y1 = f (x1 cos - x2 sin),  y2 = f (x2 cos + x1 sin)  for the pairs (i, i + r/2) or (2i, 2i + 1)
             of the first r elements; the gradient is the transposed map
    4 bits   groups of 32 elements: s = bf16(amax / 7), code = 8 + rint(x / s), standing for (code - 8) s
    pages    where codes, scales and bf16 rows lie, from the byte offsets of the interface
    decode   softmax(scale q K^T) V over the keys a table of pages lists, each sequence at its own length
"""
from __future__ import annotations

import numpy as np

BLOCK = 16      # keys of a block of a 4-bit page


def bf16_bits(x):
    """Nearest bfloat16 of float64 values, half to even, in one rounding, as uint16 (normal range; NaN and infinities kept)."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    r = np.where(np.isfinite(x), np.ldexp(np.rint(m * 256.0), e - 8), x)
    with np.errstate(over="ignore"):
        return (r.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def bf16_value(bits):
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def rope(x, pos, inv_freq, pairs: bool, factor: float = 1.0, backward: bool = False):
    """x [T, heads, d] -> float64; inv_freq float32 [r / 2], pos int [T]."""
    x = np.array(x, dtype=np.float64)
    f = np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    r = 2 * f.size
    angle = np.asarray(pos).astype(np.float64)[:, None] * f[None, :]
    c, s = factor * np.cos(angle)[:, None, :], factor * np.sin(angle)[:, None, :]
    if backward:
        s = -s
    a, b = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    x1, x2 = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
    return x


def quantise(x):
    """bf16 values [..., d] (float64) -> codes uint8 [..., d], scales uint16 (bf16 bits) [..., d / 32]."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(*x.shape[:-1], -1, 32)
    amax = np.abs(y).max(-1)
    odd = ~np.isfinite(amax)
    small = ~odd & (amax < 2.0 ** -100)
    bits = bf16_bits(np.where(odd | small, 0.0, amax) / 7.0)
    s = bf16_value(bits)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s[..., None] > 0, np.clip(np.rint(y / np.where(s > 0, s, 1.0)[..., None]), -7, 7), 0.0)
    c = np.where((odd | small)[..., None], 0.0, c)
    return (c + 8).astype(np.uint8).reshape(x.shape), np.where(odd, np.uint16(0x7FC0), bits)


def value4(codes, scales):
    c = (codes.astype(np.float64) - 8).reshape(*codes.shape[:-1], -1, 32)
    return (c * bf16_value(scales)[..., None]).reshape(codes.shape)


def page_bytes(page: int, Hkv: int, d: int, int4: bool) -> int:
    return Hkv * page * (d + d // 8 if int4 else 4 * d)


def places4(d: int):
    """Byte and nibble of K codes, bytes of K scales, and the same of V, inside a block: arrays [16, d] and [16, d / 32]."""
    g = d // 32
    r, x = np.meshgrid(np.arange(BLOCK), np.arange(d), indexing="ij")
    y, z = x // 32, x % 32
    kw, kn = r * (d // 2) + 4 * ((z // 8) * g + y), 4 * (z % 2) + z % 8 // 2
    vw = 9 * d + 128 * g * (r // 8) + 4 * g * (4 * (z // 4) + r % 8 // 2) + 2 * g * (r % 2) + 4 * (y // 2)
    vn = 4 * (y % 2) + z % 4
    r, y = np.meshgrid(np.arange(BLOCK), np.arange(g), indexing="ij")
    ks = 8 * d + 2 * ((2 * (r % 8) + r // 8) * g + y)
    vs = 17 * d + 8 * g * (r % 8 // 2) + 8 * y + 4 * (r // 8) + 2 * (r % 2)
    return (kw + kn // 2, kn % 2, ks), (vw + vn // 2, vn % 2, vs)


def write4(page, key: int, head: int, keys_per_page: int, d: int, K, V):
    """Codes and scales of one key and value (K = (codes [d], scales [d / 32])) into a page (uint8 array)."""
    at = (head * (keys_per_page // BLOCK) + key // BLOCK) * 18 * d
    r = key % BLOCK
    for (byte, high, scale), (codes, scales) in zip(places4(d), (K, V)):
        for x in range(d):
            sh = 4 * int(high[r, x])
            b = at + int(byte[r, x])
            page[b] = (int(page[b]) & ~(15 << sh) & 255) | (int(codes[x]) << sh)
        for y in range(d // 32):
            b = at + int(scale[r, y])
            page[b], page[b + 1] = int(scales[y]) & 255, int(scales[y]) >> 8


def read_pool(pool, page: int, Hkv: int, d: int, int4: bool):
    """A pool [pages, page bytes] (uint8) as K, V [pages, page, Hkv, d] float64."""
    pool = np.asarray(pool)
    P = pool.shape[0]
    if not int4:
        rows = bf16_value(pool[:, :page_bytes(page, Hkv, d, False)].copy().view(np.uint16)).reshape(P, Hkv, 2, page, d)
        return rows[:, :, 0].transpose(0, 2, 1, 3), rows[:, :, 1].transpose(0, 2, 1, 3)
    blocks = pool[:, :page_bytes(page, Hkv, d, True)].reshape(P, Hkv, page // BLOCK, 18 * d)
    out = []
    for byte, high, scale in places4(d):
        codes = (blocks[..., byte] >> (4 * high).astype(np.uint8)) & 15
        scales = blocks[..., scale].astype(np.uint16) | (blocks[..., scale + 1].astype(np.uint16) << 8)
        out.append(value4(codes, scales).reshape(P, Hkv, page, d).transpose(0, 2, 1, 3))
    return tuple(out)


def paged_decode(q, K, V, table, lens, scale: float):
    """q [B,H,d]; K, V [pages, page, Hkv, d] (read_pool); table [B, max_pages]; lens [B].  Returns dict(o [B,H,d], lse [B,H]).  Pages outside the
    pool are left out, lengths cut to what the table has room for; a sequence without keys: zeros and -inf."""
    q = np.asarray(q, dtype=np.float64)
    table, lens = np.asarray(table), np.asarray(lens)
    B, H, d = q.shape
    P, page, Hkv = K.shape[:3]
    o, lse = np.zeros((B, H, d)), np.full((B, H), -np.inf)
    for b in range(B):
        n = int(min(max(int(lens[b]), 0), table.shape[1] * page))
        j = np.arange(n)
        pg = table[b, j // page]
        live = (pg >= 0) & (pg < P)
        j, pg = j[live], pg[live]
        if not j.size:
            continue
        for h in range(H):
            kv = h // (H // Hkv)
            s = scale * (K[pg, j % page, kv] @ q[b, h])
            m = s.max()
            e = np.exp(s - m)
            o[b, h] = (e / e.sum()) @ V[pg, j % page, kv]
            lse[b, h] = m + np.log(e.sum())
    return dict(o=o, lse=lse)
