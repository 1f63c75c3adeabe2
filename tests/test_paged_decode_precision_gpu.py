"""How precise decode over pages is (paged_check.py: bounds of an element, and of all results together, that a second rounding of the weights would pass), and a
served batch whose every result is held to them."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paged_check import check_paged
from paper_2609_33916_b200 import binding as mb
from test_cache_gpu import FMT, random_pool
from test_paged_decode_gpu import Case
from test_rope_gpu import freqs, host

pytestmark = pytest.mark.gpu


def check_case(c):
    K, V = oc.read_pool(c.pool.cpu().numpy(), c.page, c.Hkv, c.d, c.fmt == "int4")
    check_paged(host(c.out), host(c.lse), host(c.q), K, V, c.table.cpu().numpy(), c.lens.cpu().numpy(), c.scale, c.fmt == "int4", 0.5 if c.fmt == "int4" else np.abs(K).max(),
                pieces=c.fmt == "bf16" and c.H // c.Hkv <= 8)


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("lens,H,Hkv,d,page", [([1500, 700, 1999, 501], 32, 8, 128, 16), ([1100, 650], 64, 4, 64, 64), ([900, 1700, 0, 1], 44, 4, 128, 32),
                                               ([600] * 20 + [3, 77], 16, 16, 64, 16)])
def test_roundings(fmt, lens, H, Hkv, d, page):
    c = Case(fmt, lens, H, Hkv, d, page, seed=40)
    c.run()
    check_case(c)


@pytest.mark.parametrize("width", [None, 40, 400])
def test_values_of_one_sign(width):
    """V's codes all above 8: sums grow over the keys, what is lost of the weights is lost of the results."""
    c = Case("int4", [1500, 700, 1999, 501], 32, 8, 128, 64, width=width, seed=41)
    v = c.pool.view(c.pages, -1, 18 * c.d)[..., 9 * c.d:17 * c.d]
    v.copy_(0x99 + (v & 0x66))
    c.run()
    check_case(c)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 1), (8, 1), (12, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_values(d, H, Hkv):
    """A value that is infinite makes its element infinite, whatever bits its weight has (a key alone: a weight of 1); the others are what they are."""
    lens = [1, 2, 3, 16, 17, 40, 130]
    c = Case("bf16", lens, H, Hkv, d, 16, scale=0.05, seed=42)
    c.run()
    want = c.out.clone()
    rows = c.pool.view(torch.bfloat16).view(c.pages, Hkv, 2, 16, d)
    for b, n in enumerate(lens):
        j = n // 2
        rows[c.table[b, j // 16].long(), :, 1, j % 16, 5] = float("inf")
        rows[c.table[b, j // 16].long(), :, 1, j % 16, d - 9] = float("-inf")
    out, _ = c.run(out=torch.zeros_like(c.out))
    assert bool(torch.isposinf(out[..., 5]).all()) and bool(torch.isneginf(out[..., d - 9]).all())
    rest = [i for i in range(d) if i not in (5, d - 9)]
    assert torch.equal(out[..., rest], want[..., rest])


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("H,Hkv,d", [(8, 2, 128), (9, 1, 64)])
def test_a_served_batch_key_by_key(fmt, H, Hkv, d):
    """Prompts, then tokens one by one through a recorded step; slots that hold no key hold random bytes.  The oracle sees the keys of the pool as they are read
    back from it."""
    B, page, width = 4, 16, 8
    rng = np.random.default_rng(17)
    pages = B * width
    table = torch.from_numpy(rng.permutation(pages).reshape(B, width).astype(np.int32)).cuda()
    cache = mb.make_cache_desc(pages, page, Hkv, d, FMT[fmt])
    pool, inv = random_pool(pages, mb.moa_cache_page_bytes(cache), 2), freqs(d)
    slot_of = lambda b, j: table.cpu().numpy()[b, j // page].astype(np.int64) * page + j % page
    past = np.array([90, 1, 15, 47])
    seq, at = np.repeat(np.arange(B), past), np.concatenate([np.arange(n) for n in past])
    gen = torch.Generator(device="cuda").manual_seed(6)
    T = len(seq)
    x = torch.randn((T, H + 2 * Hkv, d), generator=gen, device="cuda").bfloat16()
    st = x.stride()[:2]
    slots = torch.from_numpy(slot_of(seq, at)).cuda()
    qo = torch.empty((T, H, d), device="cuda", dtype=torch.bfloat16)
    mb.moa_kv_append(mb.make_append_desc(cache, T, H, q_stride=st, k_stride=st, v_stride=st), x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:],
                     torch.from_numpy(at.astype(np.int32)).cuda(), slots, inv, qo, pool)
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
    written = [(seq, at, x)]
    for _ in range(4):
        x1.copy_(torch.randn(x1.shape, generator=gen, device="cuda"))
        pos.copy_(torch.from_numpy(n.astype(np.int32)))
        slot.copy_(torch.from_numpy(slot_of(np.arange(B), n)))
        written.append((np.arange(B), n.copy(), x1.clone()))
        n += 1
        lens.copy_(torch.from_numpy(n.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        K, V = oc.read_pool(pool.cpu().numpy(), page, Hkv, d, fmt == "int4")
        # the keys and values that each step wrote are in the pool: every value, and what became of every key
        most = 0.0
        for s, j, y in written:
            p = slot_of(s, j)
            k = oc.bf16_value(oc.bf16_bits(oc.rope(host(y[:, H:H + Hkv]), j, inv.cpu().numpy(), False)))
            for got, x0 in ((K, k), (V, host(y[:, H + Hkv:]))):
                np.testing.assert_array_equal(got[p // page, p % page], oc.value4(*oc.quantise(x0)) if fmt == "int4" else x0)
            most = max(most, np.abs(K[p // page, p % page]).max())
        check_paged(host(out), host(lse), host(q1), K, V, table.cpu().numpy(), n, d ** -0.5, fmt == "int4", most / 7 if fmt == "int4" else most,
                    pieces=fmt == "bf16" and H // Hkv <= 8)
