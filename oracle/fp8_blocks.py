"""8-bit matrices with a scale for each block of 128, in float64 (test
infrastructure only).

The scale of a block is the smallest power of two 2^e, e >= -126, with
max|x| / 2^e <= R (448 for E4M3, 57344 for E5M2); a code stands for x / 2^e
rounded once to the format, to nearest even.  A block with an infinity or a
NaN has scale and codes NaN.
"""

from __future__ import annotations

import math

import numpy as np

FORMATS = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}  # mantissa bits, lowest exponent, largest


def scale_of(amax: float, fmt: str) -> float:
    if not math.isfinite(amax):
        return math.nan
    e = -126
    while math.ldexp(FORMATS[fmt][2], e) < amax:
        e += 1
    return math.ldexp(1.0, e)


def round_to(v, fmt: str) -> np.ndarray:
    """Values of the format nearest to v (|v| at most the largest), ties to even."""
    bits, low, _ = FORMATS[fmt]
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        e = np.maximum(np.frexp(v)[1] - 1, low)
        step = np.ldexp(1.0, e - bits)
        return np.rint(v / step) * step


def quantize(x, block_rows: int, fmt: str) -> tuple[np.ndarray, np.ndarray]:
    """x [R, C] -> (values of the codes [R, C], scale [ceil(C / 128), ceil(R / block_rows)])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    codes = np.empty_like(x)
    scale = np.empty((-(-cols // 128), -(-rows // block_rows)))
    for c in range(scale.shape[0]):
        for r in range(scale.shape[1]):
            at = slice(r * block_rows, (r + 1) * block_rows), slice(c * 128, (c + 1) * 128)
            s = scale[c, r] = scale_of(float(np.max(np.abs(x[at]))), fmt)
            codes[at] = round_to(x[at] / s, fmt)
    return codes, scale


def values(codes, scale, block_rows: int) -> np.ndarray:
    codes = np.asarray(codes, dtype=np.float64)
    r = np.arange(codes.shape[0]) // block_rows
    c = np.arange(codes.shape[1]) // 128
    return codes * np.asarray(scale, dtype=np.float64)[c][:, r].T


def decode(codes, fmt: str) -> np.ndarray:
    """uint8 codes -> float64."""
    if fmt == "e4m3":
        from . import e4m3

        return e4m3.decode(codes)
    # E5M2 is the upper byte of a half-precision number
    return (np.asarray(codes, dtype=np.uint16) << 8).view(np.float16).astype(np.float64)
