"""Frequencies of the rotary positions (CPU), and the transformer block with positions (GPU)."""
import math

import numpy as np
import pytest

from oracle import cache as oc
from paper_2609_33916_b200.rope import rope_frequencies


def test_frequencies():
    inv, f = rope_frequencies(64)
    assert inv.dtype == np.float32 and inv.shape == (32,) and f == 1.0 and inv[0] == 1.0
    np.testing.assert_allclose(inv, [10000.0 ** (-2 * i / 64) for i in range(32)], rtol=1e-7)
    np.testing.assert_allclose(rope_frequencies(64, scaling="linear", factor=4.0)[0], inv / 4, rtol=1e-7)
    ntk, _ = rope_frequencies(64, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and abs(ntk[-1] * 4 / inv[-1] - 1) < 1e-6 and np.all(np.diff(ntk / inv) < 0)
    yarn, f = rope_frequencies(64, scaling="yarn", factor=4.0, trained_length=4096)
    turns = 4096 * inv / (2 * math.pi)
    np.testing.assert_array_equal(yarn[turns > 32.1], inv[turns > 32.1])
    np.testing.assert_allclose(yarn[turns < 0.99], inv[turns < 0.99] / 4, rtol=1e-6)
    mid = (turns < 32) & (turns > 1)
    assert mid.any() and np.all((yarn[mid] < inv[mid]) & (yarn[mid] > inv[mid] / 4))
    assert abs(f - (0.1 * math.log(4) + 1)) < 1e-12
    assert rope_frequencies(64, scaling="yarn", factor=1.0, trained_length=10)[1] == 1.0


@pytest.mark.parametrize("kw", [dict(d_rot=7), dict(d_rot=0), dict(d_rot=64, scaling="other"), dict(d_rot=64, factor=0.0), dict(d_rot=64, base=-1.0),
                                dict(d_rot=2, scaling="ntk", factor=2.0), dict(d_rot=64, scaling="yarn", factor=2.0),
                                dict(d_rot=64, scaling="yarn", factor=2.0, trained_length=10, beta_fast=1.0, beta_slow=2.0)])
def test_frequencies_refuse(kw):
    with pytest.raises(ValueError):
        rope_frequencies(**kw)


def _block(torch, packed, rope, seed=0, at_zero=False, B=2, n=130, H=2, d=64, d_ff=256):
    from paper_2609_33916_b200.block import TransformerBlock
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    dm = H * d
    w = {k: (rnd(dm, dm) * dm ** -0.5).bfloat16() for k in ("Wq", "Wk", "Wv", "Wo")}
    w.update(W1=(rnd(d_ff, dm) * dm ** -0.5).bfloat16(), W3=(rnd(d_ff, dm) * dm ** -0.5).bfloat16(), W2=(rnd(dm, d_ff) * d_ff ** -0.5).bfloat16())
    w.update({k: (1 + 0.25 * rnd(dm)).bfloat16() for k in ("g1", "g2")})
    b = TransformerBlock(torch, B, n, H, d, d_ff, True, packed_qkv=packed, rope=rope)
    if at_zero:
        b.pos.zero_()
    w = b.prepare_weights(w)
    x, dy = rnd(B * n, dm).bfloat16(), rnd(B * n, dm).bfloat16()
    y = b.forward(x, w).clone()
    dx, grads = b.backward(x, w, dy)
    return b, x, dy, w, y, dx.clone(), {k: v.clone() for k, v in grads.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [True, False])
def test_block_at_position_zero_is_the_block_without_positions(packed):
    import torch
    inv = torch.from_numpy(rope_frequencies(64)[0]).cuda()
    plain = _block(torch, packed, None)
    turned = _block(torch, packed, inv, at_zero=True)
    # dQ's contributions are added by atomics: the gradients that come from it differ by the order of fp32 sums (bf16 halves on top: a step of 2^-8)
    assert torch.equal(plain[4], turned[4])
    for a, b in [(plain[5], turned[5])] + [(plain[6][k], turned[6][k]) for k in plain[6]]:
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -6 * float(a.float().abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("d_rot,layout,factor", [(64, 0, 1.0), (32, 1, 1.25)])
def test_block_with_positions(packed, d_rot, layout, factor):
    """Forward and gradients against the same block in 64 bits, differentiated by torch.  Every array that the block keeps is bf16: about twenty roundings
    of 2^-8 lie on the way of a gradient, random in sign: sqrt(20) 2^-8 = 1.8e-2 of its norm."""
    import torch
    B, n, H, d, d_ff = 2, 130, 2, 64, 256
    inv = torch.from_numpy(rope_frequencies(d_rot)[0]).cuda()
    b, x, dy, w, y, dx, grads = _block(torch, packed, {"inv_freq": inv, "layout": layout, "factor": factor}, seed=d_rot)
    # what the projection kept are the turned q and k
    h1 = b.h1.double().cpu().numpy()
    q = (h1 @ w["Wq"].double().cpu().numpy().T).reshape(B * n, H, d)
    ref = oc.rope(q, np.tile(np.arange(n), B), inv.cpu().numpy(), bool(layout), factor)
    got = b.q.reshape(B * n, H, d)
    assert np.linalg.norm(got.double().cpu().numpy() - ref) <= 2 * 2.0 ** -8 * np.linalg.norm(ref)
    p = {k: v.double().requires_grad_() for k, v in w.items() if k != "Wqkv"}
    X = x.double().requires_grad_()
    norm = lambda t, g: t * (t.pow(2).mean(-1, keepdim=True) + 1e-5).rsqrt() * g
    ang = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * inv.double()

    def turn(t):      # [B, H, n, d]
        r = d_rot
        u, v = (t[..., 0:r:2], t[..., 1:r:2]) if layout else (t[..., :r // 2], t[..., r // 2:r])
        parts = (factor * (u * ang.cos() - v * ang.sin()), factor * (v * ang.cos() + u * ang.sin()))
        return torch.cat((torch.stack(parts, -1).flatten(-2) if layout else torch.cat(parts, -1), t[..., r:]), -1)

    heads = lambda t: t.view(B, n, H, d).transpose(1, 2)
    h1 = norm(X, p["g1"])
    Q, K, V = turn(heads(h1 @ p["Wq"].T)), turn(heads(h1 @ p["Wk"].T)), heads(h1 @ p["Wv"].T)
    s = (Q @ K.transpose(-1, -2)) / math.sqrt(d)
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -math.inf)
    x2 = X + (s.softmax(-1) @ V).transpose(1, 2).reshape(B * n, H * d) @ p["Wo"].T
    h2 = norm(x2, p["g2"])
    out = x2 + (torch.nn.functional.silu(h2 @ p["W1"].T) * (h2 @ p["W3"].T)) @ p["W2"].T
    out.backward(dy.double())
    far = lambda a, r: float((a.double() - r).norm() / r.norm())
    assert far(y, out.detach()) <= 1.8e-2
    assert far(dx, X.grad) <= 1.8e-2
    for k in p:
        assert far(grads[k], p[k].grad) <= 1.8e-2, k
