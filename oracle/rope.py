"""fp64 reference for rotary positions: the pairs of a row as complex numbers times e^(i angle).

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot_dim, base=1e4, scaling="none", factor=1.0, original_length=0.0, slow_turns=0.0, fast_turns=0.0):
    """Radians a token of every pair, one after another."""
    out = []
    for i in range(rot_dim // 2):
        f = base ** (-2.0 * i / rot_dim)
        turns = original_length * f / (2.0 * math.pi)
        if scaling == "none":
            keep = 1.0
        elif scaling == "linear":
            keep = 0.0
        elif scaling == "turns":
            keep = min(max((turns - slow_turns) / (fast_turns - slow_turns), 0.0), 1.0)
        else:
            def at(n):
                return rot_dim / 2.0 * math.log(original_length / (2.0 * math.pi * n), base)
            lo, hi = max(math.floor(at(fast_turns)), 0), min(math.ceil(at(slow_turns)), rot_dim - 1)
            keep = 1.0 - min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
        out.append(keep * f + (1.0 - keep) * f / factor)
    return np.array(out)


def turn(x, positions, freqs, offset=0, interleaved=False, magnitude=1.0):
    """Rows x [T, H, d] in fp64 with the pairs turned by positions [T]."""
    y = np.array(x, dtype=np.float64, copy=True)
    n = len(freqs)
    for i in range(n):
        a, b = (offset + 2 * i, offset + 2 * i + 1) if interleaved else (offset + i, offset + n + i)
        z = (y[..., a] + 1j * y[..., b]) * (magnitude * np.exp(1j * np.asarray(positions, dtype=np.float64) * freqs[i]))[:, None]
        y[..., a], y[..., b] = z.real, z.imag
    return y
