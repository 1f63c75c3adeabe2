"""Keys at the two ends of bf16: subnormal ones, and such that parts of the rotation leave the range of fp32 where their sum does not.  The stored key is the
nearest bf16 of the rotation in 64 bits there, too: every element."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33916_b200 import binding as mb
from test_rope_gpu import freqs, host

pytestmark = pytest.mark.gpu


def nearest_bf16(y):
    """Nearest bfloat16 of float64 values, half to even, subnormal numbers and overflow to infinity included, as uint16."""
    _, e = np.frexp(np.where(np.isfinite(y), y, 0.0))
    e = np.maximum(e - 8, -133)                   # exponent of the last place
    r = np.where(np.isfinite(y), np.ldexp(np.rint(np.ldexp(y, -e)), e), y)
    with np.errstate(over="ignore"):
        return (r.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("end,factor", [("low", 1.0), ("low", 0.75), ("high", 1.0), ("high", 1.25), ("high", 3.0)])
def test_rounding_at_the_ends(end, factor, pairs):
    T, Hkv, d = 4096, 8, 128
    rng = np.random.default_rng(11)
    # bit patterns: subnormal and the least normal numbers; the two largest binades
    mag = rng.integers(0, 3 << 7, (T, Hkv, d)) if end == "low" else rng.integers(0x7E80, 0x7F80, (T, Hkv, d))
    bits = (mag | rng.integers(0, 2, mag.shape) << 15).astype(np.uint16)
    k = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    pos, inv = torch.from_numpy(rng.integers(0, 1 << 20, T, dtype=np.int32)).cuda(), freqs(d)
    pool = torch.zeros((T // 64, Hkv, 2, 64, d), device="cuda", dtype=torch.bfloat16)
    desc = mb.make_append_desc(mb.make_cache_desc(T // 64, 64, Hkv, d), T, 0, layout=int(pairs), factor=factor)
    mb.moa_kv_append(desc, None, k, k, pos, torch.arange(T, device="cuda"), inv, None, pool)
    want = nearest_bf16(oc.rope(oc.bf16_value(bits), pos.cpu().numpy(), inv.cpu().numpy(), pairs, factor))
    got = pool[:, :, 0].transpose(1, 2).reshape(T, Hkv, d).contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    values = pool[:, :, 1].transpose(1, 2).reshape(T, Hkv, d)
    assert torch.equal(values.view(torch.int16), k.view(torch.int16))
    assert int(np.sum(got != want)) == 0, np.argwhere(got != want)[:5]
