"""Decode attention over pages against the 64-bit oracle.

Tolerance of an element, with A = sum_j p_j |v_j| of its column: the weights are rounded to bf16 (2^-8 of each; the 4-bit form may round once more where
they meet the scale), and the result is rounded to bf16: (1 or 2) 2^-8 A + 2^-8 |o|.  Scores: products are exact, and are summed in 32 bits; a sum of N
terms, each addition cut to 24 bits, is within N 2^-23 sum |terms|, in the 4-bit form of 34 terms of up to 143 |q| s per group (room for
codes that carry 128 and start from -136; those of the kernel are 1 to 15 and start from -8): e = scale 34 2^-23 (143 + 136) s sum|q|, in the bf16 form e = scale 128 2^-23 sum |q k|.  A score that is off by e
takes the weights off by a factor within 1 +- 2 e and lse by e.  fp32 sums of the weights and of the products: 1e-5."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33916_b200 import binding as mb

pytestmark = pytest.mark.gpu
FMT = {"bf16": mb.MOA_CACHE_BF16, "int4": mb.MOA_CACHE_INT4}


def host(t):
    return t.detach().double().cpu().numpy()


def make_pool(rng, fmt, pages, page, Hkv, d, stride=None):
    """Bytes of a pool with N(0,1)-like contents in every key."""
    size = oc.page_bytes(page, Hkv, d, fmt == "int4")
    if fmt == "bf16":
        raw = (rng.standard_normal((pages, size // 2)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16).view(np.uint8)
    else:
        raw = rng.integers(0, 256, (pages, Hkv, page // 16, 18 * d), dtype=np.uint8)
        s = rng.uniform(0.1, 0.5, (pages, Hkv, page // 16, 2, d // 2)).astype(np.float32)
        s = (s.view(np.uint32) >> 16).astype(np.uint16).view(np.uint8)
        raw[..., 8 * d:9 * d], raw[..., 17 * d:] = s[..., 0, :], s[..., 1, :]
        raw = raw.reshape(pages, size)
    if stride:
        raw = np.concatenate((raw, np.full((pages, stride - size), 0xFF, np.uint8)), 1)
    return torch.from_numpy(np.ascontiguousarray(raw)).cuda()


class Case:
    def __init__(self, fmt, lens, H, Hkv, d, page, width=None, scale=None, stride=0, seed=0, table=None, pages=None):
        rng = np.random.default_rng(seed)
        self.fmt, self.H, self.Hkv, self.d, self.page = fmt, H, Hkv, d, page
        self.B = len(lens)
        self.width = width or max(1, -(-max(lens) // page))
        self.pages = pages or self.B * self.width
        self.scale = d ** -0.5 if scale is None else scale
        self.pool = make_pool(rng, fmt, self.pages, page, Hkv, d, stride)
        self.table = torch.from_numpy((rng.permutation(self.pages)[:self.B * self.width].reshape(self.B, self.width) if table is None else np.asarray(table)).astype(np.int32)).cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = torch.from_numpy(rng.standard_normal((self.B, H, d))).cuda().bfloat16()
        self.cache = mb.make_cache_desc(self.pages, page, Hkv, d, FMT[fmt], stride)
        self.desc = mb.make_paged_decode_desc(self.cache, self.B, H, self.width, self.scale)
        self.ws = torch.full((mb.moa_paged_decode_workspace_bytes(self.desc),), 0xFF, dtype=torch.uint8, device="cuda")
        self.out = torch.full((self.B, H, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((self.B, H), float("nan"), device="cuda")

    def run(self, **kw):
        a = dict(q=self.q, pool=self.pool, table=self.table, lens=self.lens, out=self.out, lse=self.lse, ws=self.ws)
        a.update(kw)
        mb.moa_paged_decode(self.desc, a["q"], a["pool"], a["table"], a["lens"], a["out"], a["lse"], a["ws"])
        assert mb.moa_last_device_status() == mb.MOA_OK
        return a["out"], a["lse"]

    def check(self, out=None, lse=None, rows=None):
        out, lse = host(self.out if out is None else out), host(self.lse if lse is None else lse)
        K, V = oc.read_pool(self.pool.cpu().numpy(), self.page, self.Hkv, self.d, self.fmt == "int4")
        q, table, lens = host(self.q), self.table.cpu().numpy(), self.lens.cpu().numpy()
        if rows is not None:
            q, table, lens, out, lse = (x[rows] for x in (q, table, lens, out, lse))
        ref = oc.paged_decode(q, K, V, table, lens, self.scale)
        mass = oc.paged_decode(q, K, np.abs(V), table, lens, self.scale)["o"]
        sq = np.abs(q).sum(-1)
        if self.fmt == "int4":
            e = abs(self.scale) * 34 * 2.0 ** -23 * 279 * 0.5 * sq
        else:
            e = abs(self.scale) * 128 * 2.0 ** -23 * 5.0 * sq
        e = np.where(np.isfinite(ref["lse"]), e, 0.0)
        tol = ((2 if self.fmt == "int4" else 1) * 2.0 ** -8 + 2 * e[..., None] + 1e-5) * mass + 2.0 ** -8 * np.abs(ref["o"])
        over = np.abs(out - ref["o"]) - tol
        assert np.all(over <= 0), (float(np.nanmax(over)), np.argwhere(~(over <= 0))[:5])
        fin = np.isfinite(ref["lse"])
        np.testing.assert_array_equal(lse[~fin], ref["lse"][~fin])
        assert np.all(np.abs(lse - ref["lse"])[fin] <= (e + 1e-5 * (1 + np.abs(ref["lse"])))[fin])
        # and as a whole, what the roundings come to on average
        if fin.any() and np.linalg.norm(ref["o"]) > 0:
            assert np.linalg.norm(out - ref["o"]) <= 5e-3 * np.linalg.norm(mass)


EDGES = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200]


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv,page", [(1, 1, 16), (4, 2, 64), (8, 1, 32), (12, 3, 48), (9, 1, 16), (16, 1, 128), (7, 1, 16), (30, 2, 16)])
def test_lengths_and_groups(fmt, d, H, Hkv, page):
    c = Case(fmt, EDGES, H, Hkv, d, page, seed=H)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("lens,H,Hkv,d,page", [([5000], 32, 8, 128, 16), ([1000], 16, 16, 64, 16), ([20000, 3], 4, 1, 128, 64), ([1], 1, 1, 64, 16),
                                               ([0], 4, 2, 128, 16), ([777, 0, 0, 4097], 10, 2, 64, 1024), ([9000, 100], 24, 2, 128, 32)])
def test_shared_sequences(fmt, lens, H, Hkv, d, page):
    c = Case(fmt, lens, H, Hkv, d, page, seed=3)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("B", [127, 128, 129, 300])
def test_many_sequences(fmt, B):
    lens = np.random.default_rng(B).integers(0, 150, B).tolist()
    c = Case(fmt, lens, 4, 2, 64, 16, width=10, seed=B)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_same_result_every_time(fmt):
    c = Case(fmt, [3000, 10, 700], 8, 2, 128, 16, seed=1)
    a = [t.clone() for t in c.run()]
    for _ in range(5):
        c.ws.fill_(0xFF)
        b = c.run(out=torch.full_like(c.out, float("nan")), lse=torch.full_like(c.lse, float("nan")))
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    without = torch.empty_like(c.out)
    mb.moa_paged_decode(c.desc, c.q, c.pool, c.table, c.lens, without, None, c.ws)
    assert torch.equal(without, a[0])


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_lies_past_the_end_does_not_count(fmt, d):
    """All bytes of a pool that no sequence's keys use are made not-a-number: the same bits come out."""
    lens = [1, 17, 30, 64, 79, 100, 0]
    c = Case(fmt, lens, 4, 2, d, 16, width=8, seed=2)
    want = [t.clone() for t in c.run()]
    pool, table = c.pool.cpu().numpy().copy(), c.table.cpu().numpy()
    used = np.zeros((c.pages, c.page), bool)
    for b, n in enumerate(lens):
        j = np.arange(n)
        used[table[b, j // c.page], j % c.page] = True
    if fmt == "bf16":
        rows = pool.view(np.uint16).reshape(c.pages, 2, 2, c.page, d)
        rows[np.broadcast_to(~used[:, None, None, :, None], rows.shape)] = 0x7FC0
    else:
        blocks = pool.reshape(c.pages, 2, 18 * d)
        (kb, _, ks), (vb, _, vs) = oc.places4(d)
        for p in range(c.pages):
            for r in np.nonzero(~used[p])[0]:
                blocks[p][:, np.concatenate((kb[r], vb[r]))] = 0xFF
                for s in (ks[r], vs[r]):
                    blocks[p][:, s], blocks[p][:, s + 1] = 0xC0, 0x7F
    got = c.run(pool=torch.from_numpy(pool).cuda(), out=torch.full_like(c.out, float("nan")), lse=torch.full_like(c.lse, float("nan")))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_bad_tables_and_lengths(fmt):
    """Pages outside the pool are left out, lengths are cut: nothing is read out of bounds (the oracle does the same)."""
    lens = [300, 40, -7, 2 ** 31 - 1, -2 ** 31, 96, 5]
    rng = np.random.default_rng(4)
    table = rng.integers(0, 40, (7, 8))
    table[0, 3], table[0, 6], table[1, 0], table[5] = -1, 40, 2 ** 31 - 1, -2 ** 31
    table[6, 1:] = 10 ** 9          # (past the end)
    c = Case(fmt, lens, 4, 2, 128, 16, width=8, table=table, pages=40, seed=4)
    c.run()
    c.check()
    assert float(c.out[5].abs().max()) == 0 and bool(torch.isneginf(c.lse[5]).all())


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales(fmt, scale):
    c = Case(fmt, [130, 70], 4, 1, 64, 16, scale=scale, seed=5)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_strides(fmt):
    d, H, Hkv, page = 128, 4, 2, 32
    size = oc.page_bytes(page, Hkv, d, fmt == "int4")
    c = Case(fmt, [100, 33], H, Hkv, d, page, stride=size + 4096, seed=6)
    c.run()
    c.check()
    want = [t.clone() for t in (c.out, c.lse)]
    wide = torch.zeros((2, H + 3, d), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:H + 1] = c.q
    table = torch.full((2, c.width + 5), 10 ** 9, dtype=torch.int32, device="cuda")
    table[:, :c.width] = c.table
    c.desc = mb.make_paged_decode_desc(c.cache, 2, H, c.width, c.scale, table_stride=c.width + 5, q_stride=wide.stride()[:2])
    got = c.run(q=wide[:, 1:], table=table, out=torch.full_like(c.out, float("nan")), lse=torch.full_like(c.lse, float("nan")))
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_large_scores_and_a_query_that_is_not_a_number(fmt):
    c = Case(fmt, [400, 90], 8, 2, 128, 16, scale=1.0, seed=7)
    c.run()
    c.check()
    want = c.out.clone()
    c.q[1, 5] = float("nan")
    out, lse = c.run(out=torch.zeros_like(c.out))
    assert bool(torch.isnan(out[1, 5]).all()) and bool(torch.isnan(lse[1, 5]))
    keep = torch.ones((2, 8), dtype=torch.bool)
    keep[1, 5] = False
    assert torch.equal(out[keep], want[keep])


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_pages_past_32_bits(fmt):
    """A pool of more than 4 GB, its last and first pages in a table."""
    page, Hkv, d, H = 64, 8, 128, 16
    size = oc.page_bytes(page, Hkv, d, fmt == "int4")
    pages = (9 << 29) // size + 1
    few = make_pool(np.random.default_rng(8), fmt, 3, page, Hkv, d)
    c = Case(fmt, [150, 64], H, Hkv, d, page, width=3, pages=6, seed=8)
    c.pool = torch.cat((few, few.flip(0)))
    big = torch.empty((pages, size), dtype=torch.uint8, device="cuda")
    big[-3:], big[0] = few, few[2]
    c.table = torch.tensor([[0, 1, 2], [2, 0, 0]], dtype=torch.int32, device="cuda")
    want = [t.clone() for t in c.run()]
    c.check()
    where = torch.tensor([[pages - 3, pages - 2, 0], [pages - 1, 0, 0]], dtype=torch.int32, device="cuda")
    c.desc = mb.make_paged_decode_desc(mb.make_cache_desc(pages, page, Hkv, d, FMT[fmt]), 2, H, 3, c.scale)
    got = c.run(pool=big, table=where, out=torch.full_like(c.out, float("nan")), lse=torch.full_like(c.lse, float("nan")))
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_two_streams_with_a_workspace_each(fmt):
    a, b = Case(fmt, [5000, 300], 8, 2, 128, 16, seed=9), Case(fmt, [70, 4000], 8, 2, 128, 16, seed=10)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        for c, st in ((a, s), (b, t)):
            mb.moa_paged_decode(c.desc, c.q, c.pool, c.table, c.lens, c.out, c.lse, c.ws, stream=st)
    torch.cuda.synchronize()
    a.check()
    b.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_captured_and_replayed_with_other_lengths(fmt):
    c = Case(fmt, [2000, 2000, 2000], 8, 2, 64, 16, seed=11)
    c.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2):
            mb.moa_paged_decode(c.desc, c.q, c.pool, c.table, c.lens, c.out, c.lse, c.ws)
    for lens in ([1, 0, 2000], [1999, 17, 640], [0, 0, 0], [64, 64, 64]):
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.out.fill_(float("nan"))
        c.ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        c.check()


def test_both_formats_agree_on_what_four_bits_can_hold():
    """Keys and values that are whole multiples of their scales: the bf16 pool and the 4-bit pool hold the same numbers."""
    B, H, Hkv, d, page, n = 2, 8, 2, 128, 16, 90
    four = Case("int4", [n, 33], H, Hkv, d, page, seed=12)
    four.pool.view(four.pages, Hkv, 18 * d)[..., 8 * d:9 * d].view(torch.bfloat16)[:] = 0.25      # (code - 8) / 4: exact in bf16
    four.pool.view(four.pages, Hkv, 18 * d)[..., 17 * d:].view(torch.bfloat16)[:] = 0.5
    K, V = oc.read_pool(four.pool.cpu().numpy(), page, Hkv, d, True)
    rows = np.stack((K, V)).transpose(1, 3, 0, 2, 4)
    wide = Case("bf16", [n, 33], H, Hkv, d, page, seed=12)
    wide.pool = torch.from_numpy(np.ascontiguousarray(rows)).cuda().bfloat16().view(torch.uint8).reshape(four.pages, -1)
    wide.table, wide.q = four.table, four.q
    four.run()
    wide.run()
    four.check()
    wide.check()
    assert float((four.lse - wide.lse).abs().max()) <= 1e-4
