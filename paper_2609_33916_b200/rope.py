"""Frequencies for the rotary positions (moa_rope_fwd, moa_kv_append): a host-side table of d_rot / 2 numbers and one factor.

    plain     inv_freq[i] = base^(-2 i / d_rot)
    "linear"  positions divided by `factor`: inv_freq / factor
    "ntk"     a larger base, base * factor^(d_rot / (d_rot - 2)): the lowest frequency is divided by the factor, the highest stays
    "yarn"    by how often a pair turns over the length that was trained on: pairs that turn more than beta_fast times stay, pairs that turn less than
              beta_slow times are divided by the factor, those between are blended, linearly in the number of turns (the published form; where a model
              was trained with a ramp in the pair's index, between rounded limits, its frequencies are passed to the kernels as they are); the
              rotated q and k are multiplied by 0.1 ln(factor) + 1
"""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(d_rot: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0, trained_length: int | None = None,
                     beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(inv_freq float32 [d_rot / 2], factor of the rotated elements).  `trained_length` is wanted by "yarn"."""
    if d_rot < 2 or d_rot % 2:
        raise ValueError("d_rot must be even and positive")
    if not factor > 0 or not base > 0:
        raise ValueError("base and factor must be positive")
    i = np.arange(0, d_rot, 2, dtype=np.float64) / d_rot
    if scaling is None:
        return (base ** -i).astype(np.float32), 1.0
    if scaling == "linear":
        return (base ** -i / factor).astype(np.float32), 1.0
    if scaling == "ntk":
        if d_rot == 2:
            raise ValueError("a single pair has no lowest frequency to scale")
        return ((base * factor ** (d_rot / (d_rot - 2.0))) ** -i).astype(np.float32), 1.0
    if scaling == "yarn":
        if not trained_length or not beta_fast > beta_slow:
            raise ValueError("yarn wants trained_length, and beta_fast above beta_slow")
        plain = base ** -i
        turns = trained_length * plain / (2 * math.pi)
        keep = np.clip((turns - beta_slow) / (beta_fast - beta_slow), 0.0, 1.0)
        return (plain * keep + plain / factor * (1 - keep)).astype(np.float32), 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    raise ValueError(f"unknown scaling {scaling!r}")
