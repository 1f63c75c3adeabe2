"""What the results of paged decode are held to, tighter than a maximum over the pool: used by the tests of its precision, of its range and of served batches.

Of an element, with A = sum_j p_j |v_j| of its column and p the normalised weights:
  weights   bf16 pages, groups of 9 to 16: a weight is rounded once, 2^-8 A; smaller groups (`pieces`): a weight is a bf16 below it and a rest of 2^-7 at most, which is
            rounded: 2^-15 A, and twice as many sums, 1e-5 A.  4 bits: its product with V's scale is, 2^-8 A; the product comes from two pieces, of which the
            smaller, 2^-7 at most, is rounded itself and again with the scale: 2 * 2^-15 A.
  result    rounded to bf16: 2^-8 |o|
  scores    products are exact and summed in fp32, each addition cut to 24 bits: N terms are within N 2^-23 sum |terms|.  4 bits: 32 products of codes up to
            15 and two parts of the starting value -8 sum(q), per group, 34 * 2^-23 (15 + 8) s sum|q|, and the groups' sum, four roundings of at most
            8 s sum|q|: e = scale s sum|q| 2^-23 (34 * 23 + 16); bf16: e = scale 128 * 2^-23 sum|q k|.  A score that is off by e takes a normalised weight off by
            a factor within 1 +- 2 e, and lse by e.
  the rest  the argument of a weight's power is at most 128 in size and is rounded to 24 bits, 2^-18, the power itself is within 2^-22; sums of 2000 keys, 16 at once
            in each of four warps: 32 * 2^-23; joins: a few 2^-24: 1e-5 A together.
Of the results of many long rows together, each as a part of its norm: a rounding is off by 2^(e-8) / 3^0.5 in the mean square, where the number is m 2^e with m in
[1, 2).  Where logarithms are spread evenly, the mean square of m is 3 / (2 ln 2), so of the numbers' own it is 2^-8 (2 ln 2 / 9)^0.5 = 1.53e-3.  Values of both
signs: the weights' errors add up as the results themselves do.  Two roundings, the weight's or its product's and the result's, are 2.17e-3, three 2.66e-3: the bound
lies between, at 2.45 of them, 2.40e-3 (in pieces: one rounding, 1.45 of them, 1.85e-3), and holds rows of 500 keys and more, where there are 64 at least."""
import numpy as np

from oracle import cache as oc

ONE = 2.0 ** -8 * (2 * np.log(2) / 9) ** 0.5


def check_paged(out, lse, q, K, V, table, lens, scale, four_bits, most_key, low=0.0, pieces=False):
    """out, lse: the results (float64).  most_key: the largest K scale (4 bits) or |k|.  low: what an element may be off by besides."""
    ref = oc.paged_decode(q, K, V, table, lens, scale)
    mass = oc.paged_decode(q, K, np.abs(V), table, lens, scale)["o"]
    sq = np.abs(q).sum(-1)
    e = abs(scale) * 2.0 ** -23 * (34 * 23 + 16 if four_bits else 128) * most_key * sq
    fin = np.isfinite(ref["lse"])
    e = np.where(fin, e, 0.0)
    weights = 2.0 ** -15 + 1e-5 if pieces else 2.0 ** -8 + (2 * 2.0 ** -15 if four_bits else 0.0)
    tol = (weights + 2 * e[..., None] + 1e-5) * mass + 2.0 ** -8 * np.abs(ref["o"]) + low
    over = np.abs(out - ref["o"]) - tol
    assert np.all(over <= 0), (float(np.nanmax(over / (mass + 1e-300))), np.argwhere(~(over <= 0))[:5])
    np.testing.assert_array_equal(lse[~fin], ref["lse"][~fin])
    assert np.all(np.abs(lse[fin] - ref["lse"][fin]) <= (e + 1e-5 * (1 + np.abs(np.where(fin, ref["lse"], 0.0))))[fin])
    long = np.broadcast_to((np.asarray(lens) >= 500)[:, None], fin.shape) & fin
    if long.sum() >= 64:
        far = np.linalg.norm(out - ref["o"], axis=-1)[long] / np.linalg.norm(ref["o"], axis=-1)[long]
        assert np.sqrt(np.mean(far ** 2)) <= ((1.45 if pieces else 2.45) ** 0.5) * ONE, np.sqrt(np.mean(far ** 2))
    return ref
