"""Rotary positions on the GPU against the 64-bit oracle, element by element.

Tolerance of an element: the rounding of the result, half a step (bf16 2^-8, fp32 2^-24 of it), and what 32-bit arithmetic adds: cosine and
sine 1.5 * 2^-24, the factor, the products and their sum 2^-24 each: at most 4.5 * 2^-24 < 4e-7 of f (|x1| + |x2|)."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_33916_b200 import binding as mb

pytestmark = pytest.mark.gpu
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def freqs(d_rot, base=10000.0):
    return torch.from_numpy((base ** (-np.arange(0, d_rot, 2) / d_rot)).astype(np.float32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def reference(x, pos, inv, pairs, factor, backward):
    """The oracle's result, and the tolerance."""
    x, r = host(x), 2 * inv.numel()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    y = oc.rope(x, pos.cpu().numpy(), inv.cpu().numpy(), pairs, factor, backward)
    both = np.zeros_like(x)
    both[..., a] = both[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, both * 4e-7 * abs(factor), r


def check(got, x, pos, inv, pairs, factor=1.0, backward=False):
    y, tol, r = reference(x, pos, inv, pairs, factor, backward)
    g = host(got)
    assert np.all(np.abs(g - y) <= tol + ROUND[got.dtype] * np.abs(y)), np.max(np.abs(g - y) - tol - ROUND[got.dtype] * np.abs(y))
    np.testing.assert_array_equal(g[..., r:], host(x)[..., r:])


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype,T,H,Hk,d,d_rot", [
    (torch.bfloat16, 1, 1, 1, 64, 64), (torch.bfloat16, 7, 4, 2, 128, 128), (torch.bfloat16, 1001, 3, 1, 128, 64), (torch.bfloat16, 33, 5, 0, 256, 256),
    (torch.bfloat16, 130, 2, 2, 80, 32), (torch.bfloat16, 65, 3, 2, 72, 72), (torch.bfloat16, 9, 2, 1, 8, 8), (torch.bfloat16, 40, 7, 3, 96, 40),
    (torch.bfloat16, 3, 300, 4, 64, 16), (torch.bfloat16, 2500, 1, 1, 128, 112), (torch.float32, 1, 2, 1, 128, 128), (torch.float32, 301, 4, 2, 80, 32),
    (torch.float32, 17, 3, 1, 256, 248), (torch.float32, 1300, 1, 1, 64, 64), (torch.bfloat16, 5, 2, 1, 256, 248), (torch.float32, 6, 2, 0, 8, 8)])
def test_against_the_oracle(dtype, T, H, Hk, d, d_rot, pairs, backward):
    gen = torch.Generator(device="cuda").manual_seed(T + d)
    q, k = (torch.randn((T, h, d), generator=gen, device="cuda").to(dtype) for h in (H, max(Hk, 1)))
    pos = torch.randint(0, 200000, (T,), generator=gen, device="cuda", dtype=torch.int32)
    inv = freqs(d_rot)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    desc = mb.make_rope_desc(T, H, Hk, d, d_rot, int(pairs), 1.25, mb.MOA_BF16 if dtype == torch.bfloat16 else mb.MOA_F32)
    call = mb.moa_rope_bwd if backward else mb.moa_rope_fwd
    call(desc, pos, inv, q, k if Hk else None, qo, ko if Hk else None)
    check(qo, q, pos, inv, pairs, 1.25, backward)
    if Hk:
        check(ko, k, pos, inv, pairs, 1.25, backward)
    else:
        assert torch.isnan(ko).all()
    # in place: the same bits
    q2, k2 = q.clone(), k.clone()
    call(desc, pos, inv, q2, k2 if Hk else None, q2, k2 if Hk else None)
    assert torch.equal(q2, qo) and (not Hk or torch.equal(k2, ko))


@pytest.mark.parametrize("T", [5, 700])
def test_parts_of_a_packed_projection(T):
    """q and k rotated in place inside [T, H + 2 Hk, d]; v, and a head-major output, beside them."""
    H, Hk, d = 6, 2, 128
    x = torch.randn((T, H + 2 * Hk, d), device="cuda").bfloat16()
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    inv, before = freqs(d), x.clone()
    st = x.stride()[:2]
    desc = mb.make_rope_desc(T, H, Hk, d, q_stride=st, k_stride=st, q_out_stride=st, k_out_stride=st)
    mb.moa_rope_fwd(desc, pos, inv, x[:, :H], x[:, H:H + Hk], x[:, :H], x[:, H:H + Hk])
    check(x[:, :H], before[:, :H], pos, inv, False)
    check(x[:, H:H + Hk], before[:, H:H + Hk], pos, inv, False)
    assert torch.equal(x[:, H + Hk:], before[:, H + Hk:])
    out = torch.full((H, T + 3, d), float("nan"), device="cuda").bfloat16()
    desc = mb.make_rope_desc(T, H, 0, d, q_stride=st, q_out_stride=(d, (T + 3) * d))
    mb.moa_rope_fwd(desc, pos, inv, before, None, out, None)
    assert torch.equal(out[:, :T].transpose(0, 1), x[:, :H]) and torch.isnan(out[:, T:]).all()


def test_far_and_negative_positions():
    T, d = 64, 128
    x = torch.randn((T, 2, d), device="cuda")
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, -10 ** 6, 123456789] * 8, dtype=torch.int32, device="cuda")
    inv, y = freqs(d), torch.empty_like(x)
    mb.moa_rope_fwd(mb.make_rope_desc(T, 2, 0, d, dtype=mb.MOA_F32), pos, inv, x, None, y, None)
    # (the product of position and frequency has up to 55 bits and a double 53: 2^31 radians are exact to 2^-22, half of it in the product, half in the
    # reduction, and the oracle's product rounds the same way)
    g, (ref, tol, _) = host(y), reference(x, pos, inv, False, 1.0, False)
    far = np.where(np.abs(pos.cpu().numpy()) > 1e8, 2.0 ** -21, 0.0)[:, None, None]
    assert np.all(np.abs(g - ref) <= tol + 2.0 ** -24 * np.abs(ref) + far * tol / 4e-7)


@pytest.mark.parametrize("pairs", [False, True])
def test_gradients(pairs):
    """The backward call against the gradient of the definition, and against differences of the forward call."""
    T, H, d, r, f = 37, 3, 64, 48, 0.75
    x, dy = (torch.randn((T, H, d), device="cuda") for _ in range(2))
    pos, inv = torch.randint(0, 5000, (T,), device="cuda", dtype=torch.int32), freqs(r)
    desc = mb.make_rope_desc(T, H, 0, d, r, int(pairs), f, mb.MOA_F32)
    dx = torch.empty_like(x)
    mb.moa_rope_bwd(desc, pos, inv, dy, None, dx, None)
    leaf = x.double().requires_grad_()
    ang = pos.double()[:, None, None] * inv.double()
    a, b = (leaf[..., 0:r:2], leaf[..., 1:r:2]) if pairs else (leaf[..., :r // 2], leaf[..., r // 2:r])
    parts = (f * (a * ang.cos() - b * ang.sin()), f * (b * ang.cos() + a * ang.sin()))
    y = torch.cat(((torch.stack(parts, -1).flatten(-2) if pairs else torch.cat(parts, -1)), leaf[..., r:]), -1)
    (y * dy.double()).sum().backward()
    assert float((dx.double() - leaf.grad).abs().max()) <= 4e-7 * 2 * float(dy.abs().max())
    # the map is linear: a difference of any size is the derivative
    v = torch.randn_like(x)
    y0, y1 = torch.empty_like(x), torch.empty_like(x)
    mb.moa_rope_fwd(desc, pos, inv, x, None, y0, None)
    mb.moa_rope_fwd(desc, pos, inv, x + v, None, y1, None)
    lhs, rhs = float(((y1.double() - y0.double()) * dy.double()).sum()), float((dx.double() * (x + v).double().sub(x.double())).sum())
    n = x.numel()
    assert abs(lhs - rhs) <= n * 4 * 4e-7 * 2 * float(dy.abs().max()) * float((x.abs() + v.abs()).max())


def test_not_numbers_stay_with_their_pair():
    T, H, d = 3, 2, 64
    x = torch.randn((T, H, d), device="cuda").bfloat16()
    x[1, 0, 5], x[2, 1, 40] = float("nan"), float("inf")
    y = torch.empty_like(x)
    mb.moa_rope_fwd(mb.make_rope_desc(T, H, 0, d), torch.arange(T, device="cuda", dtype=torch.int32), freqs(d), x, None, y, None)
    odd = ~torch.isfinite(y)
    assert odd.nonzero().tolist() == [[1, 0, 5], [1, 0, 37], [2, 1, 8], [2, 1, 40]]


def test_streams_and_graphs():
    T, H, Hk, d = 50, 4, 2, 128
    q, k = torch.randn((T, H, d), device="cuda").bfloat16(), torch.randn((T, Hk, d), device="cuda").bfloat16()
    pos, inv = torch.arange(T, device="cuda", dtype=torch.int32), freqs(d)
    desc = mb.make_rope_desc(T, H, Hk, d)
    want = torch.empty_like(q), torch.empty_like(k)
    mb.moa_rope_fwd(desc, pos, inv, q, k, *want)
    torch.cuda.synchronize()
    side, out = torch.cuda.Stream(), (torch.empty_like(q), torch.empty_like(k))
    with torch.cuda.stream(side):
        mb.moa_rope_fwd(desc, pos, inv, q, k, *out)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    back = torch.empty_like(q), torch.empty_like(k)
    with torch.cuda.graph(graph):
        mb.moa_rope_fwd(desc, pos, inv, q, k, *out)
        mb.moa_rope_bwd(desc, pos, inv, *out, *back)
    q.copy_(torch.randn_like(q))
    graph.replay()
    torch.cuda.synchronize()
    check(out[0], q, pos, inv, False)
    check(back[0], out[0], pos, inv, False, 1.0, True)
