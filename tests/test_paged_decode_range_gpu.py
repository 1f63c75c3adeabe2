"""Decode over 4-bit pages whose numbers are small or large: codes are used at the low end of bf16, so sums of weights and values, and of queries and codes,
lie near the low end of fp32.

What the sums' last place stands for: an accumulator of O is 2^-69 (half of the elements: 2^-65) of its value, so fp32's last place 2^-149 is 2^-80 there: a result
is off by at most 2^-80 for each product of 16 keys, for the joins of four warps and for moving the reference (the weights' sum is 1 at least): (n / 16 + 8) 2^-80.
A group's product with a query is 2^-65 of its value: three roundings (two products, the starting value) of 2^-84, times K's scale, in each of d / 32 groups."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paged_check import check_paged
from test_paged_decode_gpu import Case, host

pytestmark = pytest.mark.gpu


def scale_pool(c, k_exp, v_exp):
    """K's and V's scales times 2^k_exp and 2^v_exp, exactly (bf16 exponents)."""
    blocks = c.pool.view(c.pages, -1, 18 * c.d)
    for at, e in ((8, k_exp), (17, v_exp)):
        s = blocks[..., at * c.d:(at + 1) * c.d].view(torch.bfloat16)
        s.copy_((s.double() * 2.0 ** e).bfloat16())


@pytest.mark.parametrize("d,H,Hkv", [(64, 4, 2), (128, 8, 2), (128, 12, 1)])
@pytest.mark.parametrize("v_exp", [54, 20, -40, -56, -60, -66, -72, -76])
def test_values_of_any_size(d, H, Hkv, v_exp):
    """v_exp 54: values just below 2^55.  Lengths of one (no reference moved) and of many."""
    lens = [1, 2, 5, 300, 0, 1500]
    c = Case("int4", lens, H, Hkv, d, 16, scale=0.3, seed=30)
    scale_pool(c, 0, v_exp - 2 if v_exp > 0 else v_exp)
    c.run()
    K, V = oc.read_pool(c.pool.cpu().numpy(), c.page, Hkv, d, True)
    assert np.abs(V).max() < 2.0 ** 55
    low = (max(lens) / 16 + 8) * 2.0 ** -80
    ref = check_paged(host(c.out), host(c.lse), host(c.q), K, V, c.table.cpu().numpy(), np.array(lens), c.scale, True, 0.5, low=low)
    assert v_exp < -72 or np.abs(ref["o"]).max() > 8 * low


@pytest.mark.parametrize("q_exp,k_exp,log_scale", [(56, 0, -57), (56, -56, -1), (-20, 20, -1), (-56, 56, -1), (-62, 62, -1), (-70, 70, -1), (-50, 0, 49)])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_of_any_size(d, q_exp, k_exp, log_scale):
    lens, H, Hkv = [1, 2, 5, 300, 0, 1500], 8, 2
    c = Case("int4", lens, H, Hkv, d, 16, scale=d ** -0.5 * 2.0 ** log_scale, seed=31)
    scale_pool(c, k_exp, 0)
    c.q.copy_((c.q.double().clamp(-4, 4) * 2.0 ** q_exp).bfloat16())
    c.run()
    K, V = oc.read_pool(c.pool.cpu().numpy(), c.page, Hkv, d, True)
    # the roundings of small products, as a part of a score: into the bound through the largest key
    extra = 3 * 2.0 ** -84 * (d // 32) / np.abs(host(c.q)).sum(-1).min() / (2.0 ** -23 * (34 * 23 + 16))
    check_paged(host(c.out), host(c.lse), host(c.q), K, V, c.table.cpu().numpy(), np.array(lens), c.scale, True, (0.5 + 0.5 * extra) * 2.0 ** k_exp)
