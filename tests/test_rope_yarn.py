"""The blend between the two ends of "yarn": linear in the number of turns over the trained length."""
import math

import numpy as np
import pytest

from paper_2609_33916_b200.rope import rope_frequencies


@pytest.mark.parametrize("d_rot,base,factor,length,fast,slow", [(64, 10000.0, 4.0, 4096, 32.0, 1.0), (128, 500000.0, 8.0, 8192, 32.0, 1.0), (96, 10000.0, 16.0, 2048, 20.0, 2.0)])
def test_every_frequency_of_the_blend(d_rot, base, factor, length, fast, slow):
    got, _ = rope_frequencies(d_rot, base, "yarn", factor, length, fast, slow)
    between = 0
    for i in range(d_rot // 2):
        plain = base ** (-2.0 * i / d_rot)
        turns = length * plain / (2 * math.pi)
        keep = 1.0 if turns >= fast else 0.0 if turns <= slow else (turns - slow) / (fast - slow)
        between += 0.0 < keep < 1.0
        # half a step of fp32, and a few of 64 bits
        assert abs(float(got[i]) - (keep * plain + (1 - keep) * plain / factor)) <= (2.0 ** -24 + 1e-14) * plain
    assert between >= 3 and got.dtype == np.float32
