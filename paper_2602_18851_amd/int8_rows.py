"""Matrices of 8-bit integers with a scale for each row, and their products.

``quantize_int8`` and ``matmul_int8`` check torch tensors and pass them to spectral_quantize_int8 and
spectral_matmul_int8 (include/spectral.h) on the current stream of the tensors' device.  Autograd does not record them:
a tensor that requires gradients, a matrix's scale and a given result among them, is refused unless these are off
(torch.no_grad, or inside an autograd.Function).
"""

from __future__ import annotations

import functools

import torch

from .fp8_blocks import _PLAIN, _plain
from .launch import on_stream_of, refuse_autograd
from .spectral import (SN_BF16, SN_F32, SN_I8, SN_STRIDE_ZERO, sn_matmul_int8, spectral_matmul_int8,
                       spectral_matmul_int8_workspace_bytes, spectral_quantize_int8)

_TYPES = {torch.int8: SN_I8, torch.float32: SN_F32, torch.bfloat16: SN_BF16}


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(m, n, k, a_type, c_type) -> int:
    return spectral_matmul_int8_workspace_bytes(sn_matmul_int8(m, n, k, a_type, c_type))


class Int8Matrix:
    """A matrix [rows, cols] in 8-bit integers: ``codes`` int8 [rows, >= cols rounded up to 16] (rows contiguous and
    16-byte aligned, columns past ``cols`` not used) and ``scale`` float32 [rows], any stride: element (r, c) is
    codes[r, c] * scale[r]."""

    __slots__ = ("codes", "scale", "rows", "cols", "ld")

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, cols: int | None = None):
        if codes.dtype != torch.int8 or codes.dim() != 2 or not codes.is_cuda:
            raise ValueError("codes must be a two-dimensional int8 CUDA tensor")
        rows, width = codes.shape
        if cols is None:
            cols = width
        if not 0 <= cols <= width:
            raise ValueError(f"cols must be in [0, {width}]")
        full = (cols + 15) // 16 * 16
        if width < full:
            raise ValueError("code rows must hold their columns rounded up to 16")
        step, one = codes.stride()
        self.ld = step if rows > 1 and cols else full
        if cols and (one != 1 or self.ld % 16 or self.ld < full or codes.data_ptr() % 16):
            raise ValueError("code rows must be contiguous and 16-byte aligned")
        if scale.dtype != torch.float32 or scale.device != codes.device or tuple(scale.shape) != (rows,):
            raise ValueError(f"scale must be a float32 tensor [{rows}] on the codes' device")
        self.codes, self.scale, self.rows, self.cols = codes, scale, rows, cols

    @classmethod
    def _made(cls, codes: torch.Tensor, scale: torch.Tensor, rows: int, cols: int, ld: int) -> "Int8Matrix":
        """One of the quantiser's own, which needs no checks."""
        m = object.__new__(cls)
        m.codes, m.scale, m.rows, m.cols, m.ld = codes, scale, rows, cols, ld
        return m

    @property
    def values(self) -> torch.Tensor:
        """The codes [rows, cols] without the columns that fill up their rows."""
        return self.codes[:, :self.cols]


def _scale_stride(m: Int8Matrix) -> int:
    """Zero, one value expanded over all rows, would say "dense" to the library."""
    return m.scale.stride(0) or SN_STRIDE_ZERO


def quantize_int8(x: torch.Tensor) -> Int8Matrix:
    """x [R, C] (float32 or bfloat16, row-major) to 8-bit integers: a row's scale is max|x| / 127 rounded to float32
    (2^-126 at least), a code x / scale rounded to the nearest, ties to even.  A row that holds an infinity or a NaN gets
    scale NaN and codes zero."""
    ld_x = _plain(x, "x")
    r, c = x.shape
    ld = (c + 15) // 16 * 16
    codes = torch.empty((r, ld), dtype=torch.int8, device=x.device)
    scale = torch.empty((r,), dtype=torch.float32, device=x.device)
    if r:
        on_stream_of(x.device, spectral_quantize_int8, x.data_ptr(), r, c, ld_x, _TYPES[x.dtype], codes.data_ptr(), ld,
                     scale.data_ptr())
    return Int8Matrix._made(codes, scale, r, c, ld)


def matmul_int8(a, b: Int8Matrix, out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None) -> torch.Tensor:
    """a b^T: a [M, K] an Int8Matrix, or a float32 or bfloat16 tensor that is quantised on the way; b [N, K] an
    Int8Matrix, K below 2^17.  The sums of codes are exact.  ``out``: [M, N] float32 or bfloat16, rows contiguous, apart
    from a and b.  ``workspace``: uint8 scratch for callers that keep it (a new tensor where it is too small); calls that can
    run at the same time need their own."""
    if not isinstance(b, Int8Matrix):
        raise ValueError("b must be an Int8Matrix")
    if b.scale.requires_grad:
        refuse_autograd("b.scale")
    if isinstance(a, Int8Matrix):
        if a.scale.requires_grad:
            refuse_autograd("a.scale")
        codes, ld_a, m, k, sa, sa_row = a.codes, a.ld, a.rows, a.cols, a.scale.data_ptr(), _scale_stride(a)
    else:
        codes, ld_a, sa, sa_row = a, _plain(a, "a"), 0, 0
        m, k = a.shape
    n, dev = b.rows, codes.device
    if b.cols != k:
        raise ValueError(f"a has {k} columns and b {b.cols}")
    if b.codes.device != dev:
        raise ValueError("a and b are on different devices")
    if out is None:
        if out_dtype not in _PLAIN:
            raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
        out = torch.empty((m, n), dtype=out_dtype, device=dev)
        ld_c = n
    else:
        if tuple(out.shape) != (m, n) or out.device != dev or out.dtype not in _PLAIN:
            raise ValueError(f"out must be a float32 or bfloat16 tensor [{m}, {n}] on {dev}")
        ld_c, one = out.stride()
        if (n > 1 and one != 1) or (m > 1 and ld_c < n):
            raise ValueError("out must be row-major")
        if m <= 1:
            ld_c = n
        if out.requires_grad:
            refuse_autograd("out")
    if m == 0 or n == 0:
        return out
    kinds = (m, n, k, _TYPES[codes.dtype], _TYPES[out.dtype])
    need = _workspace_bytes(*kinds)
    ws = 0
    if need:
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
        ws = workspace.data_ptr()
    p = sn_matmul_int8(*kinds, ld_a, b.ld, ld_c, sa_row, _scale_stride(b))
    on_stream_of(dev, spectral_matmul_int8, p, codes.data_ptr(), sa, b.codes.data_ptr(), b.scale.data_ptr(),
                 out.data_ptr(), ws, need)
    return out
