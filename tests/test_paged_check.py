"""What the check of paged decode's results lets through, on the CPU: the kernels' arithmetic in numpy passes, and the same with a mistake in it does not."""
import numpy as np
import pytest

from oracle import cache as oc
from paged_check import check_paged

LENS = np.array([3, 700, 600, 0, 1500, 129, 800, 900])


def to_bf16(x):
    return oc.bf16_value(oc.bf16_bits(x))


def upper_half(x):
    """fp32 values cut to bf16."""
    return (np.asarray(x, np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)


def world(four_bits, same_sign=False, seed=0):
    rng = np.random.default_rng(seed)
    pages, page, Hkv, H, d = 300, 16, 4, 16, 128
    if four_bits:
        codes = [rng.integers(1, 16, (pages, page, Hkv, d)), rng.integers(9 if same_sign else 1, 16, (pages, page, Hkv, d))]
        scales = [to_bf16(rng.uniform(0.1, 0.5, (pages, page, Hkv, d // 32))) for _ in range(2)]
        K, V = ((c - 8.0) * np.repeat(s, 32, -1) for c, s in zip(codes, scales))
        vs = np.repeat(scales[1], 32, -1)
    else:
        K, V = to_bf16(rng.standard_normal((pages, page, Hkv, d))), to_bf16(rng.standard_normal((pages, page, Hkv, d)))
        vs = None
    q = to_bf16(rng.standard_normal((len(LENS), H, d)))
    table = np.zeros((len(LENS), 100), dtype=np.int32)
    order = iter(rng.permutation(pages))
    for b, n in enumerate(LENS):
        for i in range(-(-n // page)):
            table[b, i] = next(order)
    return q, K, V, vs, table


def kernel(q, K, V, vs, table, scale, how):
    """The kernels' roundings.  how: "right", or the mistake."""
    (B, H, d), (_, page, Hkv, _) = q.shape, K.shape
    out, lse = np.zeros((B, H, d)), np.full((B, H), -np.inf)
    for b, n in enumerate(LENS):
        if n == 0:
            continue
        j = np.arange(n)
        pg = table[b, j // page]
        for h in range(H):
            kv = h // (H // Hkv)
            s = scale * (K[pg, j % page, kv] @ q[b, h])
            p = np.exp(s - s.max()).astype(np.float32).astype(np.float64)
            v = V[pg, j % page, kv]
            if how == "next value":
                v = np.roll(v, -1, 0)
            if how == "one weight for all":
                p = np.ones_like(p)
            if vs is None:
                w = upper_half(p) if how == "cut" else p if how == "in pieces" else to_bf16(p)
                o = w @ v
            else:
                f = vs[pg, j % page, kv]
                first = {"rounded twice": to_bf16, "cut": upper_half}.get(how, lambda x: x)(p)
                o = np.sum(to_bf16(first[:, None] * f) * (v / f), 0)
            out[b, h] = to_bf16(o / p.sum())
            lse[b, h] = s.max() + np.log(p.sum())
    return out, lse


@pytest.mark.parametrize("same_sign", [False, True])
def test_the_kernels_arithmetic_passes(same_sign):
    for four_bits in (False, True):
        q, K, V, vs, table = world(four_bits, same_sign)
        out, lse = kernel(q, K, V, vs, table, 0.09, "right")
        check_paged(out, lse, q, K, V, table, LENS, 0.09, four_bits, 0.5 if four_bits else 5.0)


@pytest.mark.parametrize("four_bits,how", [(True, "rounded twice"), (True, "cut"), (False, "cut"), (True, "next value"), (False, "next value"),
                                           (True, "one weight for all"), (False, "one weight for all")])
def test_mistakes_do_not(four_bits, how):
    q, K, V, vs, table = world(four_bits)
    out, lse = kernel(q, K, V, vs, table, 0.09, how)
    _, right = kernel(q, K, V, vs, table, 0.09, "right")
    with pytest.raises(AssertionError):
        check_paged(out, right, q, K, V, table, LENS, 0.09, four_bits, 0.5 if four_bits else 5.0)
    if how in ("next value", "one weight for all"):        # and these in few short rows: by the bounds of the elements alone
        b = [0, 5]
        with pytest.raises(AssertionError):
            check_paged(out[b], right[b], q[b], K, V, table[b], LENS[b], 0.09, four_bits, 0.5 if four_bits else 5.0)


def test_a_rounded_weight_is_not_one_in_pieces():
    q, K, V, vs, table = world(False)
    out, lse = kernel(q, K, V, vs, table, 0.09, "in pieces")
    check_paged(out, lse, q, K, V, table, LENS, 0.09, False, 5.0, pieces=True)
    out, lse = kernel(q, K, V, vs, table, 0.09, "right")
    with pytest.raises(AssertionError):
        check_paged(out, lse, q, K, V, table, LENS, 0.09, False, 5.0, pieces=True)


def test_a_stale_result_does_not():
    q, K, V, vs, table = world(True)
    out, lse = kernel(q, K, V, vs, table, 0.09, "right")
    out[1] = out[2]
    with pytest.raises(AssertionError):
        check_paged(out, lse, q, K, V, table, LENS, 0.09, True, 0.5)
