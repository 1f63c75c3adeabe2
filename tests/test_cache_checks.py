"""Rotary positions and the paged cache without a GPU: descriptor layouts, refusals, page sizes, and the oracle pinned by what it must satisfy
(norms, relative positions, closed forms; every place of a page used once; the bounds of the 4-bit rounding)."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import cache as oc
from oracle import decode_attn
from paper_2609_33916_b200 import binding as mb
from paper_2609_33916_b200 import build as mbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 4096      # an aligned address that is never dereferenced: the checks fail first


@pytest.fixture(scope="module", autouse=True)
def _built():
    mbuild.build()


def test_header_symbols_are_exported():
    with open(os.path.join(ROOT, "include", "moa_cache.h")) as f:
        declared = set(re.findall(r"\b(moa_[a-z_0-9]+)\s*\(", f.read()))
    assert declared == set(mb.CACHE_EXPORTS), declared ^ set(mb.CACHE_EXPORTS)
    for name in declared:
        assert hasattr(mb.lib(), name), name


def test_descriptor_layouts():
    assert [ctypes.sizeof(t) for t in (mb.moa_rope_desc, mb.moa_cache_desc, mb.moa_append_desc, mb.moa_gather_desc, mb.moa_paged_decode_desc)] == \
        [96, 32, 120, 72, 80]
    assert mb.moa_rope_desc.q_stride.offset == 32 and mb.moa_paged_decode_desc.table_stride.offset == 56


def _rope(p=(A,) * 6, **kw):
    args = dict(T=5, H=4, H_k=2, d=128)
    strides = {k: kw.pop(k) for k in list(kw) if k.endswith("stride")}
    args.update({k: kw.pop(k) for k in list(kw) if k in args})
    d = mb.make_rope_desc(*(args[k] for k in ("T", "H", "H_k", "d")), **kw, **strides)
    got = mb.moa_rope_fwd(d, *p, stream=0, check=False)
    assert mb.moa_rope_bwd(d, *p, stream=0, check=False) == got
    return got


@pytest.mark.parametrize("kw", [dict(T=0), dict(T=-1), dict(H=0), dict(H_k=-1), dict(d=0), dict(d_rot=0), dict(d_rot=136), dict(layout=2), dict(dtype=3),
                                dict(factor=float("nan")), dict(factor=float("inf")), dict(q_stride=(100, 128)), dict(q_stride=(512, 0)),
                                dict(q_stride=(516, 128)), dict(k_stride=(-256, 128)), dict(q_out_stride=(128, 128)), dict(k_out_stride=(128, 136)),
                                dict(q_stride=(1024, 128))])
def test_rope_refuses(kw):
    # (the last one: in place, with strides of the input that are not those of the output)
    assert _rope(**kw) == mb.MOA_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(d=100, d_rot=8), dict(d=264), dict(d_rot=12), dict(d_rot=4), dict(H=1 << 20)])
def test_rope_does_not_support(kw):
    assert _rope(**kw) == mb.MOA_ERR_UNSUPPORTED


def test_rope_pointers():
    for i in range(6):
        bad = [A] * 6
        bad[i] = None
        assert _rope(tuple(bad)) == mb.MOA_ERR_INVALID_ARG, i
        bad[i] = A + 2
        assert _rope(tuple(bad)) == mb.MOA_ERR_INVALID_ARG, i


CACHE = dict(pages=10, page=64, H_kv=2, d=128, format=mb.MOA_CACHE_INT4)
BAD_CACHE = [(dict(pages=0), 1), (dict(page=0), 1), (dict(H_kv=0), 1), (dict(d=-64), 1), (dict(format=2), 1), (dict(page_stride=-16), 1),
             (dict(page_stride=18432 + 8), 1), (dict(page_stride=18432 - 16), 1), (dict(page=24), 2), (dict(page=2048), 2), (dict(d=96), 2), (dict(d=256), 2)]


def _cache(**kw):
    return mb.make_cache_desc(**dict(CACHE, **kw))


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_bad_pools(kw, want):
    c = _cache(**kw)
    assert mb.moa_cache_page_bytes(c) == 0
    assert mb.moa_kv_append(mb.make_append_desc(c, 3, 4, d_rot=64), *([A] * 8), stream=0, check=False) == want
    assert mb.moa_kv_gather(mb.make_gather_desc(c, 3), *([A] * 4), stream=0, check=False) == want
    d = mb.make_paged_decode_desc(c, 2, 8, 4, 0.1)
    assert mb.moa_paged_decode_workspace_bytes(d) == 0
    assert mb.moa_paged_decode(d, *([A] * 7), stream=0, ws_bytes=1 << 40, check=False) == want
    c.reserved = 1
    assert mb.moa_cache_page_bytes(c) == 0


def test_page_bytes():
    assert mb.moa_cache_page_bytes(_cache()) == 2 * 64 * 144 == oc.page_bytes(64, 2, 128, True)
    assert mb.moa_cache_page_bytes(_cache(d=64, page=16)) == 2 * 16 * 72
    assert mb.moa_cache_page_bytes(_cache(format=mb.MOA_CACHE_BF16, page_stride=1 << 20)) == 2 * 64 * 512


@pytest.mark.parametrize("kw,want", [(dict(T=0), 1), (dict(H=-1), 1), (dict(d_rot=-16), 1), (dict(d_rot=144), 1), (dict(layout=5), 1), (dict(factor=float("nan")), 1),
                                     (dict(d_rot=0), 1), (dict(dtype=mb.MOA_F32), 2), (dict(dtype=9), 1), (dict(d_rot=24), 2), (dict(k_stride=(64, 128)), 1),
                                     (dict(q_out_stride=(128, 128)), 1), (dict(v_stride=(260, 128)), 1)])
def test_append_refuses(kw, want):
    args = dict(T=3, H=4)
    args.update(kw)
    assert mb.moa_kv_append(mb.make_append_desc(_cache(), **args), *([A] * 8), stream=0, check=False) == want


def test_append_pointers():
    d = mb.make_append_desc(_cache(), 3, 4)
    for i in range(8):
        bad = [A] * 8
        bad[i] = None
        assert mb.moa_kv_append(d, *bad, stream=0, check=False) == mb.MOA_ERR_INVALID_ARG, i
        bad[i] = A + 2
        assert mb.moa_kv_append(d, *bad, stream=0, check=False) == mb.MOA_ERR_INVALID_ARG, i


@pytest.mark.parametrize("kw,want", [(dict(B=0), 1), (dict(H=0), 1), (dict(H=7), 1), (dict(max_pages=0), 1), (dict(scale=float("inf")), 1), (dict(dtype=4), 1),
                                     (dict(table_stride=3), 1), (dict(table_stride=-4), 1), (dict(q_stride=(100, 128)), 1), (dict(H=34), 2), (dict(dtype=mb.MOA_F32), 2),
                                     (dict(max_pages=1 << 25), 2), (dict(B=1 << 28), 2), (dict(scale=1e20), 2), (dict(scale=-1e20), 2)])
def test_paged_decode_refuses(kw, want):
    args = dict(B=2, H=8, max_pages=4, scale=0.1)
    args.update(kw)
    d = mb.make_paged_decode_desc(_cache(), **args)
    assert mb.moa_paged_decode(d, *([A] * 7), stream=0, ws_bytes=1 << 40, check=False) == want
    assert mb.moa_paged_decode_workspace_bytes(d) == 0


def test_paged_decode_pointers_and_workspace():
    d = mb.make_paged_decode_desc(_cache(), 2, 8, 4, 0.1)
    need = mb.moa_paged_decode_workspace_bytes(d)
    assert 0 < need < 1 << 24
    call = lambda p, n=need: mb.moa_paged_decode(d, *p, stream=0, ws_bytes=n, check=False)
    for i in (0, 1, 2, 3, 4):
        p = [A] * 7
        p[i] = None
        assert call(p) == mb.MOA_ERR_INVALID_ARG, i
        p[i] = A + 2
        assert call(p) == mb.MOA_ERR_INVALID_ARG, i
    assert call([A] * 7, need - 1) == mb.MOA_ERR_WORKSPACE
    assert call([A] * 6 + [None]) == mb.MOA_ERR_WORKSPACE
    assert call([A] * 6 + [A + 8]) == mb.MOA_ERR_INVALID_ARG
    with pytest.raises(mb.MoaError):
        mb.moa_paged_decode(d, A, A, A, A, None, stream=0)


# ------------------------------------------------------------------------------------------------------------------ the oracle

@pytest.mark.parametrize("pairs", [False, True])
def test_oracle_rope(pairs):
    rng = np.random.default_rng(0)
    inv = (10000.0 ** (-np.arange(0, 32, 2) / 32)).astype(np.float32)
    x, y = rng.standard_normal((2, 1, 48)), rng.standard_normal((2, 1, 48))
    at = lambda v, p: oc.rope(v, np.array([p, p]), inv, pairs)
    np.testing.assert_array_equal(at(x, 0), x)
    np.testing.assert_array_equal(at(x, 7)[..., 32:], x[..., 32:])
    np.testing.assert_allclose(np.sum(at(x, 12345) ** 2), np.sum(x ** 2), rtol=1e-12)
    # the product of two rotated vectors depends on the distance alone, and the backward pass undoes the forward
    np.testing.assert_allclose(np.sum(at(x, 1003) * at(y, 1000)), np.sum(at(x, 3) * y), rtol=1e-9)
    np.testing.assert_allclose(oc.rope(at(x, 77), np.array([77, 77]), inv, pairs, backward=True), x, atol=1e-12)
    # one pair by hand
    i = 3
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + 16)
    th = 5 * float(inv[i])
    assert abs(at(x, 5)[0, 0, a] - (x[0, 0, a] * np.cos(th) - x[0, 0, b] * np.sin(th))) < 1e-14
    # the gradient is the transposed map: <rope(x), y> = <x, rope_bwd(y)>
    bwd = oc.rope(y, np.array([9, 9]), inv, pairs, 1.5, backward=True)
    np.testing.assert_allclose(np.sum(oc.rope(x, np.array([9, 9]), inv, pairs, 1.5) * y), np.sum(x * bwd), rtol=1e-12)


def test_oracle_bf16():
    torch = pytest.importorskip("torch")
    x = np.random.default_rng(1).standard_normal(10000).astype(np.float32)
    want = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    np.testing.assert_array_equal(oc.bf16_bits(x.astype(np.float64)), want)
    # one rounding: a value a hair above a tie goes up, although 32 bits would round it to the tie and then down to even
    assert oc.bf16_bits(np.float64(1.0 + 2.0 ** -8 + 2.0 ** -40)) == 0x3F81


@pytest.mark.parametrize("d", [64, 128])
def test_oracle_places_are_a_bijection(d):
    (kb, kh, ks), (vb, vh, vs) = oc.places4(d)
    nib = np.concatenate([(2 * b + h).ravel() for b, h in ((kb, kh), (vb, vh))])
    byt = np.concatenate([np.stack((s, s + 1)).ravel() for s in (ks, vs)])
    used = np.zeros(36 * d, int)
    np.add.at(used, nib, 1)
    np.add.at(used, np.stack((2 * byt, 2 * byt + 1)).ravel(), 1)
    assert np.all(used == 1)


def test_oracle_quantise():
    rng = np.random.default_rng(2)
    x = oc.bf16_value(oc.bf16_bits(rng.standard_normal((50, 128)) * np.exp(rng.standard_normal((50, 1)) * 3)))
    codes, scales = oc.quantise(x)
    s = np.repeat(oc.bf16_value(scales), 32, -1)
    assert codes.min() >= 1 and codes.max() <= 15
    # off by half a step; at the ends the scale's own rounding (2^-8) comes on top: 7 (1 + 2^-8) steps are cut to 7
    assert np.all(np.abs(oc.value4(codes, scales) - x) <= s * 0.5 * (1 + 2 ** -7))
    assert np.all(np.abs(codes.astype(int) - 8).reshape(50, 4, 32).max(-1) == 7)
    ties = np.zeros((1, 32))
    ties[0, :5] = [7.0, 2.5, 3.5, -2.5, 0.5]      # halves go to even
    assert list(oc.quantise(ties)[0][0, :5].astype(int) - 8) == [7, 2, 4, -2, 0]
    odd = np.zeros((3, 32))
    odd[0, 3], odd[1, 4], odd[2, 5] = np.nan, -np.inf, 2.0 ** -101
    c, sc = oc.quantise(odd)
    assert np.all(c == 8) and np.isnan(oc.bf16_value(sc[:2])).all() and sc[2] == 0


def test_oracle_paged_decode_is_decode_over_the_listed_keys():
    rng = np.random.default_rng(3)
    P, page, Hkv, d, H = 9, 16, 2, 64, 4
    K, V = rng.standard_normal((2, P, page, Hkv, d))
    q = rng.standard_normal((3, H, d))
    table = np.array([[3, 1, 8, 0], [2, -1, 4, 9], [5, 6, 7, 0]])
    lens = np.array([37, 64, 0])
    got = oc.paged_decode(q, K, V, table, lens, 0.3)
    keys = lambda X, rows: np.concatenate(rows)[None].transpose(0, 2, 1, 3)
    for b, rows in ((0, [(3, 16), (1, 16), (8, 5)]), (1, [(2, 16), (4, 16)])):
        ref = decode_attn(q[b:b + 1], keys(K, [K[p][:n] for p, n in rows]), keys(V, [V[p][:n] for p, n in rows]), 0.3)
        np.testing.assert_allclose(got["o"][b], ref["o"][0], atol=1e-12)
        np.testing.assert_allclose(got["lse"][b], ref["lse"][0], atol=1e-12)
    assert np.all(got["o"][2] == 0) and np.all(np.isneginf(got["lse"][2]))


@pytest.mark.parametrize("d", [64, 128])
def test_oracle_pool_round_trip(d):
    rng = np.random.default_rng(4)
    P, page, Hkv = 2, 32, 2
    pool = rng.integers(0, 256, (P, oc.page_bytes(page, Hkv, d, True)), dtype=np.uint8)
    K0, V0 = oc.read_pool(pool, page, Hkv, d, True)
    k, v = oc.bf16_value(oc.bf16_bits(rng.standard_normal((2, d))))
    oc.write4(pool[1], 21, 1, page, d, oc.quantise(k), oc.quantise(v))
    K1, V1 = oc.read_pool(pool, page, Hkv, d, True)
    np.testing.assert_array_equal(K1[1, 21, 1], oc.value4(*oc.quantise(k)))
    np.testing.assert_array_equal(V1[1, 21, 1], oc.value4(*oc.quantise(v)))
    for X in (K0, K1, V0, V1):
        X[1, 21, 1] = 0
    np.testing.assert_array_equal(K0, K1)
    np.testing.assert_array_equal(V0, V1)
