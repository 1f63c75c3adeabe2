"""What the results of paged decode are held to, tighter than a maximum over the pool: used by the tests of its precision, of its range and of served batches.

Of an element, with A = sum_j p_j |v_j| of its column and p the normalised weights:
  weights   bf16 pages: a weight is rounded once, 2^-8 A.  4 bits: its product with V's scale is, 2^-8 A; the product comes from two pieces, of which the
            smaller, 2^-7 at most, is rounded itself and again with the scale: 2 * 2^-15 A.
  result    rounded to bf16: 2^-8 |o|
  scores    products are exact and summed in fp32, each addition cut to 24 bits: N terms are within N 2^-23 sum |terms|.  4 bits: 32 products of codes up to
            15 and two parts of the starting value -8 sum(q), per group, 34 * 2^-23 (15 + 8) s sum|q|, and the groups' sum, four roundings of at most
            8 s sum|q|: e = scale s sum|q| 2^-23 (34 * 23 + 16); bf16: e = scale 128 * 2^-23 sum|q k|.  A score that is off by e takes a normalised weight off by
            a factor within 1 +- 2 e, and lse by e.
  the rest  the argument of a weight's power is at most 128 in size and is rounded to 24 bits, 2^-18, the power itself is within 2^-22; sums of 2000 keys, 16 at once
            in each of four warps: 32 * 2^-23; joins: a few 2^-24: 1e-5 A together.
Of all results together, as a part of |o|: a rounding of numbers whose logarithms are spread evenly is off by 2^-8 (0.541 / 3)^0.5 = 1.66e-3 of them in the mean
square (half a step is 2^-8 / m at m in [1, 2), and the mean of m^-2 is 3 / (8 ln 2)).  Values of both signs: weights' errors add up as the results themselves do.
Two roundings, the weight's or its product's and the result's, are 2.35e-3, three 2.87e-3: the bound is two and a half, 2.62e-3."""
import numpy as np

from oracle import cache as oc

NORM = 2.5 ** 0.5 * 1.66e-3


def check_paged(out, lse, q, K, V, table, lens, scale, four_bits, most_key, low=0.0, norm=True):
    """out, lse: the results (float64).  most_key: the largest K scale (4 bits) or |k|.  low: what an element may be off by besides."""
    ref = oc.paged_decode(q, K, V, table, lens, scale)
    mass = oc.paged_decode(q, K, np.abs(V), table, lens, scale)["o"]
    sq = np.abs(q).sum(-1)
    e = abs(scale) * 2.0 ** -23 * (34 * 23 + 16 if four_bits else 128) * most_key * sq
    fin = np.isfinite(ref["lse"])
    e = np.where(fin, e, 0.0)
    weights = 2.0 ** -8 + (2 * 2.0 ** -15 if four_bits else 0.0)
    tol = (weights + 2 * e[..., None] + 1e-5) * mass + 2.0 ** -8 * np.abs(ref["o"]) + low
    over = np.abs(out - ref["o"]) - tol
    assert np.all(over <= 0), (float(np.nanmax(over / (mass + 1e-300))), np.argwhere(~(over <= 0))[:5])
    np.testing.assert_array_equal(lse[~fin], ref["lse"][~fin])
    assert np.all(np.abs(lse[fin] - ref["lse"][fin]) <= (e + 1e-5 * (1 + np.abs(np.where(fin, ref["lse"], 0.0))))[fin])
    if norm:
        far = float(np.linalg.norm(out - ref["o"]) / np.linalg.norm(ref["o"]))
        assert far <= NORM, far
    return ref
