"""The paged cache's append and read-back on the GPU, and the whole way of a served sequence (append, decode, append ...).

K and V in the pool are compared bit by bit: the append rounds the exact rotation once, and codes and scales follow from those bits."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33916_b200 import binding as mb
from test_rope_gpu import check, freqs, host

pytestmark = pytest.mark.gpu
FMT = {"bf16": mb.MOA_CACHE_BF16, "int4": mb.MOA_CACHE_INT4}


def expected_pool(pool, fmt, page, Hkv, d, k, v, slot):
    """The pool (host bytes) after k, v [T, Hkv, d] (bf16 values) are written at slot."""
    pool = pool.copy()
    P = pool.shape[0]
    for t, s in enumerate(slot):
        if not 0 <= s < P * page:
            continue
        p, key = divmod(int(s), page)
        for h in range(Hkv):
            if fmt == "int4":
                oc.write4(pool[p], key, h, page, d, oc.quantise(k[t, h]), oc.quantise(v[t, h]))
            else:
                rows = pool[p, :oc.page_bytes(page, Hkv, d, False)].view(np.uint16).reshape(Hkv, 2, page, d)
                rows[h, 0, key], rows[h, 1, key] = oc.bf16_bits(k[t, h]), oc.bf16_bits(v[t, h])
    return pool


def random_pool(pages, stride, seed=0):
    return torch.from_numpy(np.random.default_rng(seed).integers(0, 256, (pages, stride), dtype=np.uint8)).cuda()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("layout,d,d_rot,T,H,Hkv,page,extra", [
    (0, 128, 128, 1, 4, 1, 16, 0), (0, 128, 128, 37, 8, 2, 64, 0), (1, 128, 128, 21, 4, 4, 16, 0), (0, 64, 64, 50, 2, 2, 32, 0), (1, 64, 32, 33, 6, 3, 48, 0),
    (0, 128, 64, 40, 3, 1, 16, 16), (0, 128, 32, 19, 2, 2, 16, 0), (0, 64, 48, 18, 4, 2, 16, 32), (0, 128, 16, 9, 1, 1, 32, 0), (0, 128, 112, 70, 5, 5, 16, 0),
    (1, 128, 96, 65, 1, 1, 128, 0), (0, 128, 0, 23, 0, 2, 16, 0), (0, 64, 0, 23, 0, 1, 16, 0), (0, 64, 16, 5, 0, 2, 16, 0), (0, 128, 128, 700, 1, 1, 16, 0)])
def test_append(fmt, layout, d, d_rot, T, H, Hkv, page, extra):
    rng = np.random.default_rng(T * d + d_rot)
    pages = -(-2 * T // page) + 1
    stride = oc.page_bytes(page, Hkv, d, fmt == "int4") + extra
    cache = mb.make_cache_desc(pages, page, Hkv, d, FMT[fmt], stride if extra else 0)
    x = torch.from_numpy(rng.standard_normal((T, H + 2 * Hkv, d)) * np.exp(rng.standard_normal((T, H + 2 * Hkv, 1)))).cuda().bfloat16()
    q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    pos = torch.from_numpy(rng.integers(0, 1 << 20, T, dtype=np.int32)).cuda()
    slot = rng.permutation(pages * page)[:T]
    if T > 4:
        slot[3], slot[4] = -1, pages * page          # padding, and a slot past the pool
    dslot = torch.from_numpy(slot).cuda()
    inv = freqs(d_rot) if d_rot else None
    pool = random_pool(pages, stride)
    before = pool.cpu().numpy()
    qo = torch.full((T, max(H, 1), d), float("nan"), device="cuda", dtype=torch.bfloat16)
    st = x.stride()[:2]
    desc = mb.make_append_desc(cache, T, H, d_rot, layout, 1.25 if d_rot else 1.0, q_stride=st, k_stride=st, v_stride=st)
    mb.moa_kv_append(desc, q if H else None, k, v, pos if d_rot else None, dslot, inv, qo if H else None, pool)
    if H:
        check(qo, q, pos, inv, bool(layout), 1.25)
    turned = oc.rope(host(k), pos.cpu().numpy(), inv.cpu().numpy(), bool(layout), 1.25) if d_rot else host(k)
    kb = oc.bf16_value(oc.bf16_bits(turned))
    np.testing.assert_array_equal(pool.cpu().numpy(), expected_pool(before, fmt, page, Hkv, d, kb, host(v), slot))
    # read back, also at slots that are nowhere
    for dtype, out in ((mb.MOA_F32, torch.float32), (mb.MOA_BF16, torch.bfloat16)):
        ko, vo = (torch.full((T, Hkv, d), float("nan"), device="cuda", dtype=out) for _ in range(2))
        mb.moa_kv_gather(mb.make_gather_desc(cache, T, dtype), pool, dslot, ko, vo)
        live = (slot >= 0) & (slot < pages * page)
        for got, val in ((ko, kb), (vo, host(v))):
            want = np.where(live[:, None, None], oc.value4(*oc.quantise(val)) if fmt == "int4" else val, 0.0)
            np.testing.assert_array_equal(host(got), oc.bf16_value(oc.bf16_bits(want)) if out == torch.bfloat16 else want)


def test_ties_and_borders_of_the_codes():
    """Groups with many exact ties between codes (scales that are powers of two), neighbours of ties, and ends of the range."""
    T, Hkv, d, page = 64, 2, 128, 16
    rng = np.random.default_rng(5)
    n = rng.integers(-14, 15, (T, Hkv, d)) / 2.0 * np.exp2(rng.integers(-20, 20, (T, Hkv, 1)))
    n[..., ::32] = 7.0 * np.exp2(np.floor(np.log2(np.abs(n).max(-1, keepdims=True) / 7 + 1e-30)))
    x = torch.from_numpy(n).cuda().bfloat16()
    x[::2] = (x[::2].view(torch.int16) + 1).view(torch.bfloat16)        # one step beside
    cache = mb.make_cache_desc(T // page, page, Hkv, d, mb.MOA_CACHE_INT4)
    pool = random_pool(T // page, mb.moa_cache_page_bytes(cache))
    before, slot = pool.cpu().numpy(), np.arange(T)
    mb.moa_kv_append(mb.make_append_desc(cache, T, 0, 0), None, x, x.flip(0).contiguous(), None, torch.from_numpy(slot).cuda(), None, None, pool)
    np.testing.assert_array_equal(pool.cpu().numpy(), expected_pool(before, "int4", page, Hkv, d, host(x), host(x.flip(0)), slot))


def test_not_numbers_and_small_groups():
    T, d, page = 16, 64, 16
    x = torch.randn((T, 1, d), device="cuda").bfloat16()
    x[1, 0, 3], x[2, 0, 40], x[3] = float("nan"), float("-inf"), 0.0
    x[4] *= 2.0 ** -110
    x[5, 0, :32] = 3e38
    cache = mb.make_cache_desc(1, page, 1, d, mb.MOA_CACHE_INT4)
    pool = random_pool(1, mb.moa_cache_page_bytes(cache))
    before, slot = pool.cpu().numpy(), np.arange(T)
    mb.moa_kv_append(mb.make_append_desc(cache, T, 0, 0), None, x, x, None, torch.from_numpy(slot).cuda(), None, None, pool)
    np.testing.assert_array_equal(pool.cpu().numpy(), expected_pool(before, "int4", page, 1, d, host(x), host(x), slot))


def test_rounding_of_k_is_the_nearest():
    """A few million rotated elements against the nearest bf16 of the 64-bit rotation: every one."""
    T, Hkv, d = 4096, 8, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randn((T, Hkv, d), generator=gen, device="cuda").bfloat16()
    pos = torch.randint(0, 1 << 20, (T,), generator=gen, device="cuda", dtype=torch.int32)
    inv = freqs(d)
    cache = mb.make_cache_desc(T // 64, 64, Hkv, d)
    pool = torch.zeros((T // 64, Hkv, 2, 64, d), device="cuda", dtype=torch.bfloat16)
    mb.moa_kv_append(mb.make_append_desc(cache, T, 0), None, k, k, pos, torch.arange(T, device="cuda"), inv, None, pool)
    want = oc.bf16_bits(oc.rope(host(k), pos.cpu().numpy(), inv.cpu().numpy(), False))
    got = pool[:, :, 0].transpose(1, 2).reshape(T, Hkv, d).contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    assert int(np.sum(got != want)) == 0


def test_slots_past_32_bits():
    """A pool of more than 4 GB: the last pages."""
    page, Hkv, d = 1024, 8, 128
    size = oc.page_bytes(page, Hkv, d, True)
    pages = (9 << 29) // size + 1
    pool = torch.empty((pages, size), dtype=torch.uint8, device="cuda")
    pool[-2:] = 0x88
    T = 40
    slot = torch.arange(pages * page - T, pages * page, device="cuda")
    k, v = torch.randn((2, T, Hkv, d), device="cuda").bfloat16()
    cache = mb.make_cache_desc(pages, page, Hkv, d, mb.MOA_CACHE_INT4)
    mb.moa_kv_append(mb.make_append_desc(cache, T, 0, 0), None, k, v, None, slot, None, None, pool)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    mb.moa_kv_gather(mb.make_gather_desc(cache, T), pool, slot, ko, vo)
    for got, x in ((ko, k), (vo, v)):
        np.testing.assert_array_equal(host(got), oc.bf16_value(oc.bf16_bits(oc.value4(*oc.quantise(host(x))))))
    assert bool((pool[-2] == 0x88).all())


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_a_served_batch(fmt):
    """Prompts of three sequences, then tokens one by one, the token's step captured once and replayed as the sequences grow: after every step the cache
    and the attention's result are what the definitions give."""
    B, H, Hkv, d, page, width = 3, 8, 2, 128, 16, 6
    rng = np.random.default_rng(7)
    pages = B * width
    table = torch.from_numpy(rng.permutation(pages).reshape(B, width).astype(np.int32)).cuda()
    cache = mb.make_cache_desc(pages, page, Hkv, d, FMT[fmt])
    pool = random_pool(pages, mb.moa_cache_page_bytes(cache), 1)          # (random bytes: some of them not numbers)
    inv = freqs(d)
    past = np.array([37, 1, 63])
    seq = np.repeat(np.arange(B), past)
    at = np.concatenate([np.arange(n) for n in past])
    slot_of = lambda b, j: table.cpu().numpy()[b, j // page].astype(np.int64) * page + j % page
    x = torch.randn((len(seq), H + 2 * Hkv, d), device="cuda").bfloat16()
    st, T = x.stride()[:2], len(seq)
    qo = torch.empty((T, H, d), device="cuda", dtype=torch.bfloat16)
    mb.moa_kv_append(mb.make_append_desc(cache, T, H, q_stride=st, k_stride=st, v_stride=st), x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:],
                     torch.from_numpy(at.astype(np.int32)).cuda(), torch.from_numpy(slot_of(seq, at)).cuda(), inv, qo, pool)
    # the step, over static buffers
    x1 = torch.zeros((B, H + 2 * Hkv, d), device="cuda", dtype=torch.bfloat16)
    pos, slot = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), -1, dtype=torch.int64, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    q1 = torch.empty((B, H, d), device="cuda", dtype=torch.bfloat16)
    out, lse = torch.empty_like(q1), torch.empty((B, H), device="cuda")
    app = mb.make_append_desc(cache, B, H, q_stride=st, k_stride=st, v_stride=st)
    dec = mb.make_paged_decode_desc(cache, B, H, width, d ** -0.5)
    ws = torch.full((mb.moa_paged_decode_workspace_bytes(dec),), 0xFF, dtype=torch.uint8, device="cuda")

    def step():
        mb.moa_kv_append(app, x1[:, :H], x1[:, H:H + Hkv], x1[:, H + Hkv:], pos, slot, inv, q1, pool)
        mb.moa_paged_decode(dec, q1, pool, table, lens, out, lse, ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    n = past.copy()
    for i in range(5):
        x1.copy_(torch.randn_like(x1))
        pos.copy_(torch.from_numpy(n.astype(np.int32)))
        slot.copy_(torch.from_numpy(slot_of(np.arange(B), n)))
        before = pool.cpu().numpy()
        n += 1
        lens.copy_(torch.from_numpy(n.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        kb = oc.bf16_value(oc.bf16_bits(oc.rope(host(x1[:, H:H + Hkv]), n - 1, inv.cpu().numpy(), False)))
        np.testing.assert_array_equal(pool.cpu().numpy(), expected_pool(before, fmt, page, Hkv, d, kb, host(x1[:, H + Hkv:]), slot.cpu().numpy()))
        K, V = oc.read_pool(pool.cpu().numpy(), page, Hkv, d, fmt == "int4")
        ref = oc.paged_decode(host(q1), K, V, table.cpu().numpy(), n, d ** -0.5)
        assert np.max(np.abs(host(out) - ref["o"])) <= 2.0 ** -6 * np.max(np.abs(V[np.isfinite(V)])) and np.all(np.isfinite(host(out)))
        np.testing.assert_allclose(host(lse), ref["lse"], atol=5e-3)
