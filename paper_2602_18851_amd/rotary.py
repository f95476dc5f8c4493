"""Rotary positions of queries and keys (spectral_rotary, include/spectral.h) for torch tensors."""

from __future__ import annotations

import ctypes

import torch

from .launch import on_stream_of, refuse_autograd
from .spectral import SN_BF16, SN_F32, SN_ROTARY_COPY_PADDING, sn_rotary, spectral_rotary, spectral_rotary_frequencies

_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "index": 3, "turns": 4}
_DTYPES = {torch.float32: SN_F32, torch.bfloat16: SN_BF16}


class Rotary:
    """The plan of one model: pairs of the first ``rot_dim`` elements of a head ("half": i and i + rot_dim / 2;
    "interleaved": 2 i and 2 i + 1) turn by position times base^(-2 i / rot_dim).  ``scaling`` stretches the positions
    beyond the length ``trained``: "linear", "base", "index" and "turns" as SN_ROTARY_* in include/spectral.h."""

    def __init__(self, head_dim: int, rot_dim: int | None = None, layout: str = "half", base: float = 10000.0,
                 scaling: str = "none", factor: float = 1.0, low: float = 1.0, high: float = 32.0, trained: int = 0):
        if layout not in _LAYOUTS:
            raise ValueError("layout must be 'half' or 'interleaved'")
        if scaling not in _SCALINGS:
            raise ValueError(f"scaling must be one of {', '.join(_SCALINGS)}")
        self.plan = sn_rotary(head_dim, head_dim if rot_dim is None else rot_dim, _LAYOUTS[layout], _SCALINGS[scaling],
                              base, factor, low, high, trained)
        spectral_rotary_frequencies(self.plan)  # refuses a bad plan here

    def frequencies(self) -> tuple[list[float], float]:
        """(angle per position of each pair in radians, amplitude)."""
        return spectral_rotary_frequencies(self.plan)

    def apply(self, q: torch.Tensor, k: torch.Tensor | None = None, positions: torch.Tensor | None = None,
              start: int = 0, inverse: bool = False, out=None):
        """q, k: float32 or bfloat16 [tokens, heads, head_dim], any token and head strides.  positions: int64 [tokens],
        or None: token t is at start + t; rows of tokens at negative positions (padding) are left as out holds them, and
        are the input's own, not turned, in new tensors.  inverse turns back: the gradient.  Autograd does not record the
        call: q and k that require gradients are refused unless these are off.  out: a tensor (with k: a pair) like q (and
        k), which may be the inputs themselves; new tensors if None.  Returns the turned q, or (q, k)."""
        xs = (q,) if k is None else (q, k)
        if out is None:
            outs = None
        else:
            outs = (out,) if k is None else tuple(out)
            if len(outs) != len(xs):
                raise ValueError("out must hold one tensor for q and one for k")
        d, dev, dtype = self.plan.head_dim, q.device, q.dtype
        n = q.shape[0] if q.dim() == 3 else -1
        made, fields = [], []
        for i, x in enumerate(xs):
            shape = x.shape
            if len(shape) != 3 or shape[0] != n or shape[2] != d or x.dtype != dtype or dtype not in _DTYPES \
                    or not x.is_cuda or x.device != dev:
                raise ValueError(f"q and k must be [tokens, heads, {d}] float32 or bfloat16 CUDA tensors of one type")
            if x.requires_grad:
                refuse_autograd("qk"[i])
            xt, xh, xe = x.stride()
            if outs is None:
                o = torch.empty(shape, dtype=dtype, device=dev)
                ot, oh, oe = shape[1] * d, d, 1
            else:
                o = outs[i]
                if o.shape != shape or o.dtype != dtype or o.device != dev:
                    raise ValueError("out must have the shape, type and device of its input")
                ot, oh, oe = o.stride()
            if xe != 1 or oe != 1:
                raise ValueError("heads must be contiguous")
            made.append(o)
            fields += (x.data_ptr(), o.data_ptr(), shape[1], xt, xh, ot, oh)
        if positions is not None and (positions.dtype != torch.int64 or tuple(positions.shape) != (n,)
                                      or positions.device != dev or not positions.is_contiguous()):
            raise ValueError(f"positions must be a contiguous int64 tensor [{n}] on {dev}")
        on_stream_of(dev, spectral_rotary, self.plan, _DTYPES[dtype], n, 0 if positions is None else positions.data_ptr(),
                     start, (1 if inverse else 0) | (SN_ROTARY_COPY_PADDING if outs is None else 0),
                     (ctypes.c_int64 * len(fields))(*fields), len(xs))
        return made[0] if k is None else tuple(made)
