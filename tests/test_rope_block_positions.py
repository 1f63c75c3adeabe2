"""What a block's positions may be replaced by (CPU), and that a backward pass turns back by the positions of its forward pass (GPU)."""
from types import MappingProxyType

import pytest
import torch

from paper_2609_33916_b200.block import TransformerBlock
from paper_2609_33916_b200.rope import rope_frequencies
from test_rope_block import _block


def _bare(rope=True, T=12):
    """A block without its buffers, on the CPU."""
    b = object.__new__(TransformerBlock)
    b.torch, b.T, b.device = torch, T, torch.device("cpu")
    b.rope = MappingProxyType({"inv_freq": torch.ones(4)}) if rope else None
    return b


def test_positions_are_taken():
    b = _bare()
    pos = torch.arange(12, dtype=torch.int32)
    b.pos = pos
    assert b.pos is pos


@pytest.mark.parametrize("pos", [torch.arange(12), torch.arange(12.0), torch.arange(11, dtype=torch.int32), torch.arange(13, dtype=torch.int32),
                                 torch.arange(24, dtype=torch.int32)[::2], torch.zeros((1, 12), dtype=torch.int32), torch.zeros((), dtype=torch.int32),
                                 torch.zeros(12, dtype=torch.int32, device="meta"), list(range(12)), None],
                         ids=["int64", "float", "short", "long", "strided", "matrix", "scalar", "elsewhere", "list", "none"])
def test_positions_are_refused(pos):
    b = _bare()
    b.pos = kept = torch.zeros(12, dtype=torch.int32)
    with pytest.raises(ValueError):
        b.pos = pos
    assert b.pos is kept


def test_a_block_without_positions_takes_none():
    b = _bare(rope=False)
    with pytest.raises(ValueError):
        b.pos = torch.zeros(12, dtype=torch.int32)
    assert not hasattr(b, "pos")


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [True, False])
def test_positions_replaced_behind_the_forward_pass(packed):
    inv = torch.from_numpy(rope_frequencies(64)[0]).cuda()
    b, x, dy, w, y, dx, grads = _block(torch, packed, inv)
    assert torch.equal(b.forward(x, w), y)
    b.pos = b.pos + 1000 * (torch.arange(b.T, dtype=torch.int32, device="cuda") % 7)
    dx2, grads2 = b.backward(x, w, dy)
    # dQ's contributions are added by atomics: what comes from it differs by the order of fp32 sums (a step of 2^-8)
    for u, v in [(dx, dx2)] + [(grads[k], grads2[k]) for k in grads]:
        assert float((u.float() - v.float()).abs().max()) <= 2.0 ** -6 * float(u.float().abs().max())
    # and the new ones count from the next forward pass on
    assert not torch.equal(b.forward(x, w), y)


@pytest.mark.gpu
def test_frequencies_are_the_blocks_own():
    inv = torch.from_numpy(rope_frequencies(64)[0]).cuda()
    given = {"inv_freq": inv}
    b = _block(torch, True, given)[0]
    given["inv_freq"] = inv[:2]
    assert b.rope["inv_freq"] is inv
    with pytest.raises(TypeError):
        b.rope["inv_freq"] = inv[:2]
