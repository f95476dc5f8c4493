"""A paged cache of keys and values in 8 bits and attention over it, in float64 (test infrastructure only)."""

from __future__ import annotations

import numpy as np

from . import fp8_blocks


def rows(x, fmt: str) -> tuple[np.ndarray, np.ndarray]:
    """x [..., d] -> (values of the codes, scale [...])."""
    x = np.asarray(x, dtype=np.float64)
    flat = x.reshape(-1, x.shape[-1])
    scale = np.array([fp8_blocks.scale_of(float(np.max(np.abs(r))), fmt) for r in flat])
    codes = fp8_blocks.round_to(flat / scale[:, None], fmt)
    return codes.reshape(x.shape), scale.reshape(x.shape[:-1])


def seen(length: int, drafts: int, i: int, mask, table, page: int, pages: int) -> list[int]:
    """The places that drafted token i of a sequence sees."""
    out = []
    length = min(max(length, 0), len(table) * page)
    for t in range(length):
        if not 0 <= table[t // page] < pages:
            continue
        j = t - (length - drafts)
        if j < 0 or (j <= i if mask is None else (int(mask) >> j) & 1):
            out.append(t)
    return out


def attend(q, k, v, table, lengths, masks=None, scale=None):
    """q [B, T, Hq, d]; k, v [pages, H, page, d] values; masks None, [T] or [B, T].  Returns (out, weight * |v|, the largest
    |scale q| . |k| of each row): the last two are what rounding errors are measured by."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    b_n, t_n, hq, d = q.shape
    pages, heads, page, _ = k.shape
    scale = d ** -0.5 if scale is None else scale
    out, mag, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(b_n):
        for i in range(t_n):
            mask = None if masks is None else (masks[i] if np.ndim(masks) == 1 else masks[b][i])
            at = np.array(seen(int(lengths[b]), t_n, i, mask, table[b], page, pages), dtype=int)
            if at.size == 0:
                continue
            ids, place = np.asarray(table[b])[at // page], at % page
            for h in range(hq):
                g = h // (hq // heads)
                ks, vs = k[ids, g, place], v[ids, g, place]
                s = scale * (ks @ q[b, i, h])
                with np.errstate(invalid="ignore", over="ignore"):
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[b, i, h] = w @ vs
                    mag[b, i, h] = w @ np.abs(vs)
                    reach[b, i, h] = scale * (np.abs(ks) @ np.abs(q[b, i, h])).max()
    return out, mag, reach


def weights(q, n, scale):
    """softmax(scale q) over each row's first n elements, zeros after them: attention where place j has the key and the value
    1 in element j.  q [rows, d], n [rows].  Returns (weights, the largest |scale q| of each row)."""
    q = np.asarray(q, dtype=np.float64)
    there = np.arange(q.shape[1]) < np.asarray(n)[:, None]
    s = np.where(there, scale * q, -np.inf)
    w = np.exp(s - s.max(axis=1, keepdims=True))
    return w / w.sum(axis=1, keepdims=True), np.abs(np.where(there, scale * q, 0.0)).max(axis=1)


def weights_off(reach, bf16=False):
    """How far such weights may be off, relative to themselves, of up to 32 places.  Logits: parts of q whose sum is q to 2^-26, two
    additions in the matrix cores (2^-23 each), the factor scale log2(e) (three roundings), the exponent's and the maximum's
    rounding: less than 4.5 2^-23 of `reach`.  Its power 2^-23.  Both for the weight and for the sum of the weights, which takes ten
    additions more (2^-24 each); three parts of a weight, added (2^-23 twice); the sum's reciprocal and the product with it.
    For a bf16 result weights are two parts (2^-18), and sums of more rows take 26 additions more."""
    off = (9.0 * reach + 11.0) * 2.0 ** -23
    return off + 13.0 * 2.0 ** -23 + 2.0 ** -18 if bf16 else off
