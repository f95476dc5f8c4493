"""8-bit matrices with a scale for each block of 128, and their products.

``quantize_fp8``, ``matmul_fp8`` and ``LinearFp8`` check torch tensors and pass
them to spectral_quantize_fp8 and spectral_matmul_fp8 (include/spectral.h) on
the current stream of the tensors' device; all arithmetic runs in the HIP kernels.
Gradients are calls of their own (``LinearFp8.backward``), which autograd does not record: a tensor that
requires gradients is refused unless these are off (torch.no_grad, or inside an autograd.Function).
"""

from __future__ import annotations

import functools

import torch

from .launch import on_stream_of, refuse_autograd
from .spectral import (SN_BF16, SN_E4M3, SN_E5M2, SN_F32, SN_STRIDE_ZERO, sn_matmul, spectral_matmul_fp8,
                       spectral_matmul_fp8_workspace_bytes, spectral_quantize_fp8)

BLOCK = 128
_FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_CODES = {torch.float8_e4m3fn: SN_E4M3, torch.float8_e5m2: SN_E5M2, torch.float32: SN_F32, torch.bfloat16: SN_BF16}


_FLOAT8 = (torch.float8_e4m3fn, torch.float8_e5m2)
_PLAIN = (torch.float32, torch.bfloat16)


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(m, n, k, a_type, b_type, c_type, a_rows, b_rows) -> int:
    return spectral_matmul_fp8_workspace_bytes(sn_matmul(m, n, k, a_type, b_type, c_type, a_rows, b_rows))


class Fp8Matrix:
    """A matrix [rows, cols] in 8 bits: ``codes`` [rows, >= cols rounded up to 16] (torch.float8_e4m3fn or float8_e5m2,
    rows contiguous and 16-byte aligned, columns past ``cols`` not used) and ``scale`` float32 [ceil(cols / 128), rows] (a
    scale per row and 128 columns) or [ceil(cols / 128), ceil(rows / 128)] (per 128 x 128 tile), any strides:
    element (r, c) is codes[r, c] * scale[c // 128, r or r // 128]."""

    __slots__ = ("codes", "scale", "rows", "cols", "block_rows", "ld")

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, cols: int | None = None):
        if codes.dtype not in _FLOAT8 or codes.dim() != 2 or not codes.is_cuda:
            raise ValueError("codes must be a two-dimensional float8 CUDA tensor")
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
        if scale.dtype != torch.float32 or scale.device != codes.device:
            raise ValueError("scale must be a float32 tensor on the codes' device")
        shape = tuple(scale.shape)
        kb = (cols + 127) // 128
        if shape == (kb, rows):
            self.block_rows = 1
        elif shape == (kb, (rows + 127) // 128):
            self.block_rows = BLOCK
        else:
            raise ValueError(f"scale must be [{kb}, {rows}] or [{kb}, {(rows + 127) // 128}], got {shape}")
        self.codes, self.scale, self.rows, self.cols = codes, scale, rows, cols

    @classmethod
    def _made(cls, codes: torch.Tensor, scale: torch.Tensor, rows: int, cols: int, block_rows: int) -> "Fp8Matrix":
        """One of the quantiser's own, which needs no checks."""
        m = object.__new__(cls)
        m.codes, m.scale, m.rows, m.cols, m.block_rows = codes, scale, rows, cols, block_rows
        m.ld = (cols + 15) // 16 * 16
        return m

    @property
    def values(self) -> torch.Tensor:
        """The codes [rows, cols] without the columns that fill up their rows."""
        return self.codes[:, :self.cols]


def _plain(x: torch.Tensor, name: str) -> int:
    """The row stride of a plain matrix."""
    if not isinstance(x, torch.Tensor) or x.dtype not in _PLAIN or x.dim() != 2 or not x.is_cuda:
        raise ValueError(f"{name} must be a two-dimensional float32 or bfloat16 CUDA tensor")
    if x.requires_grad:
        refuse_autograd(name)
    rows, cols = x.shape
    step, one = x.stride()
    if (cols > 1 and one != 1) or (rows > 1 and step < cols):
        raise ValueError(f"{name} must be row-major")
    return step if rows > 1 else cols


def _scale_strides(m: Fp8Matrix) -> tuple[int, int]:
    """Two zeros, one value expanded over all blocks, would say "dense" to the library."""
    strides = m.scale.stride()
    return strides if strides != (0, 0) else (SN_STRIDE_ZERO, SN_STRIDE_ZERO)


def quantize_fp8(x: torch.Tensor, tile: bool = False, rows: bool = True, cols: bool = False,
                 fmt: str = "e4m3") -> tuple[Fp8Matrix | None, Fp8Matrix | None]:
    """x [R, C] (float32 or bfloat16, row-major) to 8 bits.  Returns (the matrix, its transpose); ``rows`` and ``cols``
    say which of the two are formed, from one reading of x.  ``tile``: a scale per 128 x 128 tile instead of per row
    (of the transpose: per column) and 128 elements."""
    ld = _plain(x, "x")
    if fmt not in _FORMATS:
        raise ValueError("fmt must be 'e4m3' or 'e5m2'")
    if not (rows or cols):
        raise ValueError("rows and cols are both false")
    r, c = x.shape
    dev, dtype = x.device, _FORMATS[fmt]

    block_rows = BLOCK if tile else 1

    def room(n, k):  # n code rows of k columns
        codes = torch.empty((n, (k + 15) // 16 * 16), dtype=dtype, device=dev)
        scale = torch.empty(((k + 127) // 128, (n + 127) // 128 if tile else n), dtype=torch.float32, device=dev)
        return Fp8Matrix._made(codes, scale, n, k, block_rows)

    a = room(r, c) if rows else None
    b = room(c, r) if cols else None
    _quantize_into(x, ld, dtype, tile, a, b)
    return a, b


def _quantize_into(x, ld, dtype, tile, a, b) -> None:
    """x and its transpose into the quantiser's own matrices a and b (or None)."""
    r, c = x.shape
    if r and c:
        ra = (a.codes.data_ptr(), a.ld, a.scale.data_ptr()) if a is not None else (0, 0, 0)
        cb = (b.codes.data_ptr(), b.ld, b.scale.data_ptr()) if b is not None else (0, 0, 0)
        on_stream_of(x.device, spectral_quantize_fp8, x.data_ptr(), r, c, ld, _CODES[x.dtype], _CODES[dtype],
                     1 if tile else 0, *ra, *cb)


def matmul_fp8(a, b: Fp8Matrix, out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """a b^T: a [M, K] an Fp8Matrix, or a float32 or bfloat16 tensor that is quantised by rows to E4M3 on the way; b
    [N, K] an Fp8Matrix.  A float32 result sums exact products in float32; for a bfloat16 one the matrix cores may add them in
    eights, each kept to 2^-13 of its eight's largest (include/spectral.h).  Scales: any whose products of one of a and one
    of b lie between 2^-126 and the largest float32.  ``out``: [M, N] float32 or bfloat16, rows contiguous, apart from a
    and b.  ``workspace``: uint8 scratch for callers that keep it (a new tensor where it is too small); calls that can run at
    the same time need their own."""
    if not isinstance(b, Fp8Matrix):
        raise ValueError("b must be an Fp8Matrix")
    plain = not isinstance(a, Fp8Matrix)
    if plain:
        ld_a = _plain(a, "a")
        codes, sa, sa_block, sa_row, a_rows = a, 0, 0, 0, 1
        m, k = a.shape
    else:
        ld_a, codes, sa, a_rows, m, k = a.ld, a.codes, a.scale.data_ptr(), a.block_rows, a.rows, a.cols
        sa_block, sa_row = _scale_strides(a)
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
    if m == 0 or n == 0:
        return out
    kinds = (m, n, k, _CODES[codes.dtype], _CODES[b.codes.dtype], _CODES[out.dtype], a_rows, b.block_rows)
    need = _workspace_bytes(*kinds)
    ws = 0
    if need:
        if workspace is None or workspace.numel() < need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
        ws = workspace.data_ptr()
    p = sn_matmul(*kinds, ld_a, b.ld, ld_c, sa_block, sa_row, *_scale_strides(b))
    on_stream_of(dev, spectral_matmul_fp8, p, codes.data_ptr(), sa, b.codes.data_ptr(), b.scale.data_ptr(),
                 out.data_ptr(), ws, need)
    return out


class LinearFp8:
    """y = x W^T with both sides in 8 bits, and its gradients.  The weight [N, K] (float32 or bfloat16) is quantised by
    tiles, and so is its transpose for dx; ``set_weight`` does so again after an update, into the same memory, so that a
    graph of the layer's calls goes on with the new weight.  ``backward=False`` (serving) leaves the transpose out.
    Activations are quantised by rows of the matrix that sums over them; ``grad_fmt`` is the format of dy.  The weight may
    be a parameter: its gradient is what ``backward`` returns."""

    def __init__(self, weight: torch.Tensor, grad_fmt: str = "e4m3", backward: bool = True):
        if grad_fmt not in _FORMATS:
            raise ValueError("grad_fmt must be 'e4m3' or 'e5m2'")
        self.grad_fmt, self._back = grad_fmt, bool(backward)
        self.weight, self.weight_t = quantize_fp8(weight.detach(), tile=True, cols=self._back)

    def set_weight(self, weight: torch.Tensor) -> None:
        """A new weight of the same shape, on the same device."""
        weight = weight.detach()
        ld, w = _plain(weight, "weight"), self.weight
        if tuple(weight.shape) != (w.rows, w.cols) or weight.device != w.codes.device:
            raise ValueError(f"weight must be [{w.rows}, {w.cols}] on {w.codes.device}")
        _quantize_into(weight, ld, _FORMATS["e4m3"], True, w, self.weight_t)

    def forward(self, x: torch.Tensor, keep: bool = False, out_dtype: torch.dtype = torch.bfloat16):
        """x [M, K] -> y [M, N].  With ``keep``: (y, what backward needs of x)."""
        if not keep:
            return matmul_fp8(x, self.weight, out_dtype)
        rows, cols = quantize_fp8(x, cols=True)
        return matmul_fp8(rows, self.weight, out_dtype), cols

    def backward(self, dy: torch.Tensor, kept: Fp8Matrix, dx_dtype: torch.dtype = torch.bfloat16,
                 dw_dtype: torch.dtype = torch.float32) -> tuple[torch.Tensor, torch.Tensor]:
        """dy [M, N] and forward's ``kept`` -> (dx [M, K], dW [N, K])."""
        if self.weight_t is None:
            raise ValueError("the layer was made with backward=False")
        rows, cols = quantize_fp8(dy, cols=True, fmt=self.grad_fmt)
        return matmul_fp8(rows, self.weight_t, dx_dtype), matmul_fp8(cols, kept, dw_dtype)
