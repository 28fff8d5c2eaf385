"""Oracle for rotary positions.  TEST INFRASTRUCTURE ONLY.

Pair by pair in float64, each pair a complex number z = a + i b times amplitude * exp(i position f):
channels (j, j + r / 2) or (2 j, 2 j + 1) of the first r.
"""
from __future__ import annotations

import numpy as np


def rope(x, positions, freq, layout: str = "half", amplitude: float = 1.0, backward: bool = False):
    """x [T, H, D] float64.  Returns (y, the sum of magnitudes |A| (|a| + |b|) behind each element: its rounding errors'
    scale; 0 where an element is copied)."""
    x = np.asarray(x, np.float64)
    y, scale = x.copy(), np.zeros_like(x)
    r = 2 * len(freq)
    for j, f in enumerate(freq):
        a, b = (j, j + r // 2) if layout == "half" else (2 * j, 2 * j + 1)
        w = amplitude * np.exp(1j * np.asarray(positions, np.float64) * f * (-1 if backward else 1))
        z = (x[..., a] + 1j * x[..., b]) * w[:, None]
        y[..., a], y[..., b] = z.real, z.imag
        scale[..., a] = scale[..., b] = abs(amplitude) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, scale
