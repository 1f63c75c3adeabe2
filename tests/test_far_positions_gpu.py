"""Positions over the whole range of int32: the angles that the rotation makes, and the rounding of the keys that rests on them.

The definition's angle is the 64-bit product of position and frequency.  With x1 = 1, x2 = 0 and a factor of 1 the results are the kernel's cosine and sine
themselves: sincospif is documented within 1 ulp (2^-24 below 1), and the correction behind it rounds once more (2^-25): 1.5 * 2^-24.  What the correction
leaves out is half the square of 2 pi 2^-26, 2^-47."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33916_b200 import binding as mb
from test_rope_gpu import freqs, host

pytestmark = pytest.mark.gpu
ENDS = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, -2 ** 31 + 1, 2 ** 30, -2 ** 30, 2 ** 28 + 1, -2 ** 28 - 1, 2 ** 26 - 1]


def positions(T, low, high):
    """T positions whose size is between 2^low and 2^high, of both signs, the ends of the range among them."""
    rng = np.random.default_rng(low)
    p = np.exp2(rng.uniform(low, high, T)).astype(np.int64) * rng.choice([-1, 1], T)
    p[:len(ENDS)] = ENDS
    return torch.from_numpy(p.clip(-2 ** 31, 2 ** 31 - 1).astype(np.int32)).cuda()


@pytest.mark.parametrize("low,high", [(0, 20), (20, 26), (26, 29), (29, 31)])
@pytest.mark.parametrize("backward", [False, True])
def test_cosine_and_sine(low, high, backward):
    T, d = 4000, 128
    pos, inv = positions(T, low, high), freqs(d)
    x = torch.zeros((T, 1, d), device="cuda")
    x[..., :d // 2] = 1.0
    y = torch.full_like(x, float("nan"))
    (mb.moa_rope_bwd if backward else mb.moa_rope_fwd)(mb.make_rope_desc(T, 1, 0, d, dtype=mb.MOA_F32), pos, inv, x, None, y, None)
    err = np.abs(host(y) - oc.rope(host(x), pos.cpu().numpy(), inv.cpu().numpy(), False, 1.0, backward))
    assert err.max() <= (1.5 + 2.0 ** -20) * 2.0 ** -24, err.max() * 2.0 ** 24


@pytest.mark.parametrize("pairs", [False, True])
def test_rounding_of_far_keys_is_the_nearest(pairs):
    """Four million rotated elements against the nearest bf16 of the 64-bit rotation: every one."""
    T, Hkv, d = 4096, 8, 128
    gen = torch.Generator(device="cuda").manual_seed(4)
    k = torch.randn((T, Hkv, d), generator=gen, device="cuda").bfloat16()
    pos, inv = positions(T, 28, 31), freqs(d, 1.2)            # (frequencies near 1: every angle is a far one)
    pool = torch.zeros((T // 64, Hkv, 2, 64, d), device="cuda", dtype=torch.bfloat16)
    mb.moa_kv_append(mb.make_append_desc(mb.make_cache_desc(T // 64, 64, Hkv, d), T, 0, layout=int(pairs)), None, k, k, pos, torch.arange(T, device="cuda"), inv, None, pool)
    want = oc.bf16_bits(oc.rope(host(k), pos.cpu().numpy(), inv.cpu().numpy(), pairs))
    got = pool[:, :, 0].transpose(1, 2).reshape(T, Hkv, d).contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    assert int(np.sum(got != want)) == 0
