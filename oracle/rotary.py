"""Rotary positions in float64 (test infrastructure only): a pair (x0, x1) is
the complex number x0 + i x1, turned by exp(i p f)."""

from __future__ import annotations

import math

import numpy as np


def frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                high: float = 32.0, trained: int = 0) -> tuple[np.ndarray, float]:
    """Angle per position of each pair, and the amplitude."""
    amplitude = 1.0
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        divided = 0.0
        if scaling == "linear":
            divided = 1.0
        elif scaling == "index":
            def index(turns):
                return rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))

            a, b = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rot - 1)
            divided = min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0)
            amplitude = 1 + 0.1 * math.log(factor)
        elif scaling == "turns":
            turns = trained * f / (2 * math.pi)
            divided = 1 - min(max((turns - low) / (high - low), 0.0), 1.0)
        out.append(f * (1 - divided) + f / factor * divided)
    return np.array(out), amplitude


def rotate(x, positions, rot: int, layout: str, freq, amplitude: float, inverse: bool = False) -> np.ndarray:
    """x [tokens, heads, head_dim] -> the same shape, float64."""
    x = np.array(x, dtype=np.float64)
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(freq)
    turn = amplitude * np.exp((-1j if inverse else 1j) * angle)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    z = (x[..., a] + 1j * x[..., b]) * turn
    x[..., a], x[..., b] = z.real, z.imag
    return x
