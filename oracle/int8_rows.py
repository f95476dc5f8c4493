"""8-bit integers with a scale for each row, in float64 (test infrastructure only).

A row's scale is max|x| / 127 rounded to float32, 2^-126 at least; a code is the whole number nearest
to x / scale, ties to even, found with exact fractions.  A row with an infinity or a NaN has scale NaN and codes zero.
"""

from __future__ import annotations

import math
from fractions import Fraction

import numpy as np


def quantize(x) -> tuple[np.ndarray, np.ndarray]:
    """x [R, C] -> (codes [R, C], scale [R], a float32's value)."""
    x = np.asarray(x, dtype=np.float64)
    codes, scale = np.zeros(x.shape), np.empty(x.shape[0])
    for r, row in enumerate(x):
        top = float(np.max(np.abs(row), initial=0.0))
        if not math.isfinite(top):
            scale[r] = math.nan
            continue
        # a quotient by 127 is never next to a tie of float32, so rounding it twice is rounding it once
        scale[r] = max(float(np.float32(top / 127.0)), 2.0 ** -126)
        near = row / scale[r]
        codes[r] = np.rint(near)
        half = np.abs(np.abs(near - np.trunc(near)) - 0.5) < 2.0 ** -40 * 127  # where the quotient's own rounding may matter
        for c in np.flatnonzero(half):
            q = Fraction(float(row[c])) / Fraction(float(scale[r]))
            low = math.floor(q)
            rest = q - low
            codes[r, c] = low + (1 if rest > Fraction(1, 2) or (rest == Fraction(1, 2) and low % 2) else 0)
    return codes, scale
