"""Paged decode where the work of one head is split: several clusters for a head, equal shares with a head over many of them, and the lengths around which
one takes over from the other; two recorded calls; drawn shapes.  Cases, oracle and tolerances as in test_paged_decode_gpu.py."""
import numpy as np
import pytest
import torch

from paper_2609_33916_b200 import binding as mb
from test_paged_decode_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("lens,H,Hkv,d,page", [([60001], 1, 1, 128, 64), ([50017], 8, 1, 128, 16), ([40000], 16, 1, 64, 128), ([40000], 11, 1, 128, 48),
                                               ([30000, 0], 8, 1, 64, 16), ([17, 45000], 4, 1, 128, 1024), ([20000, 1, 0], 4, 2, 128, 64)])
def test_few_heads_and_long_caches(fmt, lens, H, Hkv, d, page):
    c = Case(fmt, lens, H, Hkv, d, page, seed=20)
    a = [t.clone() for t in c.run()]
    c.check()
    c.ws.fill_(0xFF)
    b = c.run(out=torch.full_like(c.out, float("nan")), lse=torch.full_like(c.lse, float("nan")))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("width", [1, 4, 16, 64, 200, 600])
def test_short_sequences_in_wide_tables(fmt, width):
    """What is chosen goes by the room in the tables, the work by the lengths: parts of clusters, and clusters, that have no key."""
    c = Case(fmt, [min(width * 64, 70), 1, 0], 8, 2, 128, 64, width=width, seed=21)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("H,Hkv", [(8, 8), (8, 2)])
@pytest.mark.parametrize("B", [1, 5, 12, 19, 37])
def test_from_clusters_to_shares(fmt, H, Hkv, B):
    lens = np.random.default_rng(B).integers(1500, 2500, B).tolist()
    c = Case(fmt, lens, H, Hkv, 128, 64, seed=B)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_two_recorded_calls_with_one_workspace(fmt):
    """One after the other on a stream, a workspace is free when a call is done."""
    a, b = Case(fmt, [4000, 300], 8, 2, 128, 16, seed=9), Case(fmt, [30000], 8, 1, 128, 16, seed=10)
    ws = a.ws if a.ws.numel() > b.ws.numel() else b.ws
    graphs = []
    for c in (a, b):
        c.run(ws=ws)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            mb.moa_paged_decode(c.desc, c.q, c.pool, c.table, c.lens, c.out, c.lse, ws)
    for c in (a, b):
        c.out.fill_(float("nan"))
    for _ in range(10):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    a.check()
    b.check()


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
@pytest.mark.parametrize("seed", range(12))
def test_drawn(fmt, seed):
    rng = np.random.default_rng(1000 + seed)
    Hkv, d, page = int(rng.integers(1, 9)), int(rng.choice([64, 128])), 16 * int(rng.integers(1, 9))
    H, B = Hkv * int(rng.integers(1, 17)), int(rng.integers(1, 9))
    lens = np.exp(rng.uniform(0, np.log(6000), B)).astype(int).tolist()
    c = Case(fmt, lens, H, Hkv, d, page, scale=float(rng.uniform(0.02, 0.2)), seed=seed)
    c.run()
    c.check()
