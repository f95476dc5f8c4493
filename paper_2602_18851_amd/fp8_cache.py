"""A paged cache of keys and values in 8 bits, and attention over it.

``Fp8Cache`` checks torch tensors and passes them to spectral_cache_write, spectral_cache_read and spectral_cache_attend
(include/spectral.h) on the current stream of the cache's device.  Autograd does not record the calls: a tensor that requires
gradients, the cache's own and a given result among them, is refused unless these are off.
"""

from __future__ import annotations

import functools

import torch

from .launch import on_stream_of, refuse_autograd
from .spectral import (SN_BF16, SN_E4M3, SN_E5M2, SN_F32, sn_attend, sn_cache, spectral_cache_attend,
                       spectral_cache_attend_workspace_bytes, spectral_cache_read, spectral_cache_write)

_FORMATS = {torch.float8_e4m3fn: SN_E4M3, torch.float8_e5m2: SN_E5M2}
_NAMES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_DTYPES = {torch.float32: SN_F32, torch.bfloat16: SN_BF16}


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(heads, page, head_dim, fmt, dtype, batch, drafts, q_heads, table_cols) -> int:
    return spectral_cache_attend_workspace_bytes(
        sn_cache(None, None, None, None, 1, heads, page, head_dim, fmt),
        sn_attend(dtype, batch, drafts, q_heads, table_cols, 1.0, drafts * q_heads * head_dim, q_heads * head_dim, head_dim,
                  drafts * q_heads * head_dim, q_heads * head_dim, head_dim))


class Fp8Cache:
    """Keys and values of tokens in pages: ``k`` and ``v`` codes [pages, heads, page, head_dim] (torch.float8_e4m3fn or
    float8_e5m2), ``k_scale`` and ``v_scale`` float32 [pages, heads, page]: element e of a row is code[e] * scale, the scale
    a power of two from 2^-126 on, or NaN, as ``write`` makes them (others are not looked for: ``read`` multiplies by them,
    ``attend`` takes their power of two alone).  page is a power of two from 16 on, head_dim a multiple of 16 up to 256.  A
    page is contiguous; pages may lie apart (the codes' pages of keys and of values equally far, and their scales').  Slot n
    is place n % page of page n // page."""

    __slots__ = ("k", "k_scale", "v", "v_scale", "pages", "heads", "page", "head_dim", "device", "_c")

    def __init__(self, k: torch.Tensor, k_scale: torch.Tensor, v: torch.Tensor, v_scale: torch.Tensor):
        if not isinstance(k, torch.Tensor) or k.dtype not in _FORMATS or k.dim() != 4 or not k.is_cuda:
            raise ValueError("k must be a four-dimensional float8 CUDA tensor")
        pages, heads, page, dh = k.shape
        if v.dtype != k.dtype or v.shape != k.shape or v.device != k.device:
            raise ValueError("v must have the shape, type and device of k")
        for t in (k_scale, v_scale):
            if t.dtype != torch.float32 or t.shape != k.shape[:3] or t.device != k.device:
                raise ValueError(f"scales must be float32 tensors {list(k.shape[:3])} on the codes' device")
        if page < 16 or page & (page - 1) or page > 65536:
            raise ValueError("the page must be a power of two from 16 to 65536")
        if not 1 <= heads <= 65536 or heads * page >= 1 << 31:
            raise ValueError("heads must be in [1, 65536], and heads * page below 2^31")
        if dh % 16 or not 16 <= dh <= 256:
            raise ValueError("head_dim must be a multiple of 16 up to 256")
        far = []
        for x, y, room, align in ((k, v, heads * page * dh, 16), (k_scale, v_scale, heads * page, 4)):
            for t in (x, y):
                if pages and not t[0].is_contiguous():
                    raise ValueError("a page must be contiguous")
                if t.data_ptr() % 16:
                    raise ValueError("codes and scales must be 16-byte aligned")
            step = x.stride(0) if pages > 1 else room
            if pages > 1 and (y.stride(0) != step or step < room or step % align):
                raise ValueError("pages of keys and of values must lie equally far apart, in steps of 16 bytes, and must "
                                 "not overlap")
            far.append(step)
        self.k, self.k_scale, self.v, self.v_scale = k, k_scale, v, v_scale
        self.pages, self.heads, self.page, self.head_dim, self.device = pages, heads, page, dh, k.device
        self._c = sn_cache(k.data_ptr(), k_scale.data_ptr(), v.data_ptr(), v_scale.data_ptr(), pages, heads, page, dh,
                           _FORMATS[k.dtype], *far)

    @classmethod
    def empty(cls, pages: int, heads: int, page: int, head_dim: int, fmt: str = "e4m3", device="cuda") -> "Fp8Cache":
        """A cache of zeros."""
        if fmt not in _NAMES:
            raise ValueError("fmt must be 'e4m3' or 'e5m2'")
        codes = torch.zeros((2, pages, heads, page, head_dim), dtype=torch.uint8, device=device).view(_NAMES[fmt])
        scale = torch.zeros((2, pages, heads, page), dtype=torch.float32, device=device)
        return cls(codes[0], scale[0], codes[1], scale[1])

    def _no_gradients(self) -> None:
        if self.k_scale.requires_grad or self.v_scale.requires_grad or self.k.requires_grad or self.v.requires_grad:
            refuse_autograd("a tensor of the cache")

    def _slots(self, slots: torch.Tensor, n: int) -> int:
        if slots.dtype != torch.int64 or slots.shape != (n,) or slots.device != self.device \
                or not slots.is_contiguous():
            raise ValueError(f"slots must be a contiguous int64 tensor [{n}] on {self.device}")
        return slots.data_ptr()

    def _rows(self, x: torch.Tensor, name: str, dtype: torch.dtype, n: int) -> tuple[int, int, int]:
        if x.dtype != dtype or dtype not in _DTYPES or x.device != self.device \
                or x.shape != (n, self.heads, self.head_dim):
            raise ValueError(f"k and v must be float32 or bfloat16 tensors [tokens, {self.heads}, {self.head_dim}] of one "
                             f"type on {self.device}")
        if x.requires_grad:
            refuse_autograd(name)
        token, head, one = x.stride()
        if one != 1:
            raise ValueError("heads must be contiguous")
        return x.data_ptr(), token, head

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """k, v: float32 or bfloat16 [tokens, heads, head_dim], any token and head strides, to slots (int64 [tokens]): a
        row's scale is the smallest power of two, 2^-126 at least, with max|x| / scale <= 448 (e4m3) or 57344 (e5m2), a code x
        / scale rounded to nearest even; a row that holds an infinity or a NaN becomes NaN.  Tokens whose slot is not in
        [0, pages * page) are padding and not written; the other slots must differ."""
        shape = k.shape
        n = shape[0] if len(shape) == 3 else -1
        self._no_gradients()
        on_stream_of(self.device, spectral_cache_write, self._c, _DTYPES.get(k.dtype, -1), n,
                     *self._rows(k, "k", k.dtype, n), *self._rows(v, "v", k.dtype, n), self._slots(slots, n))

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, out=None):
        """(keys, values) of slots (int64 [tokens]), each [tokens, heads, head_dim]: code * scale rounded to dtype (float32 or
        bfloat16); zeros for slots outside.  out: a pair of tensors of one type, any token and head strides without
        overlaps; new ones of dtype if None."""
        shape = slots.shape
        n = shape[0] if len(shape) == 1 else -1
        self._no_gradients()
        if out is None:
            if dtype not in _DTYPES:
                raise ValueError("dtype must be torch.float32 or torch.bfloat16")
            at = self._slots(slots, n)
            k, v = (torch.empty((n, self.heads, self.head_dim), dtype=dtype, device=self.device) for _ in range(2))
        else:
            k, v = out
            at = self._slots(slots, n)
        on_stream_of(self.device, spectral_cache_read, self._c, _DTYPES.get(k.dtype, -1), n, at,
                     *self._rows(k, "k", k.dtype, n), *self._rows(v, "v", k.dtype, n))
        return k, v

    def attend(self, q: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, tree: torch.Tensor | None = None,
               scale: float | None = None, out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
        """softmax(scale q k^T) v of the last tokens of each sequence, whose keys and values the cache holds.  q: float32 or
        bfloat16 [batch, tokens, query heads, head_dim], 64 tokens at most, any strides but of the elements; query head h reads
        head h // (query heads // heads).  table: int32 [batch, pages of the longest], the pages of each sequence in order
        (a place whose page is outside [0, pages) is not seen).  lengths: int32 [batch], places of each sequence, the last
        ``tokens`` of them q's own.  A token sees all places before these, and of these those up to its own or, with ``tree``
        (int64 [tokens] or [batch, tokens]), token j where bit j of its mask is set.  Who sees nothing gets zeros.
        scale: head_dim ** -0.5 if None.  out: like q, without overlaps; workspace: uint8 scratch for callers that keep
        it (a new tensor where it is too small); calls that can run at the same time need their own."""
        dev, dtype, dh = self.device, q.dtype, self.head_dim
        shape = q.shape
        if len(shape) != 4 or dtype not in _DTYPES or q.device != dev or shape[3] != dh:
            raise ValueError(f"q must be a float32 or bfloat16 tensor [batch, tokens, query heads, {dh}] on {dev}")
        if q.requires_grad:
            refuse_autograd("q")
        self._no_gradients()
        batch, n, hq, _ = shape
        if not 1 <= n <= 64 or hq == 0 or hq % self.heads:
            raise ValueError(f"q must have 1 to 64 tokens and a multiple of {self.heads} heads")
        if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != batch or table.device != dev:
            raise ValueError(f"table must be an int32 tensor [{batch}, pages of the longest] on {dev}")
        cols = table.shape[1]
        table_ld, one = table.stride()
        if cols > 1 and one != 1:
            raise ValueError("table must be row-major")
        if batch <= 1 or cols == 0:
            table_ld = cols
        elif table_ld < cols:
            raise ValueError("table must be row-major")
        if lengths.dtype != torch.int32 or lengths.shape != (batch,) or lengths.device != dev \
                or not lengths.is_contiguous():
            raise ValueError(f"lengths must be a contiguous int32 tensor [{batch}] on {dev}")
        masks = mask_batch = 0
        if tree is not None:
            if tree.dtype != torch.int64 or tree.shape not in ((n,), (batch, n)) or tree.device != dev \
                    or (n > 1 and tree.stride(-1) != 1):
                raise ValueError(f"tree must be an int64 tensor [{n}] or [{batch}, {n}] on {dev}, rows contiguous")
            masks, mask_batch = tree.data_ptr(), tree.stride(0) if tree.dim() == 2 else 0
        q_strides = q.stride()
        if q_strides[3] != 1:
            raise ValueError("heads must be contiguous")
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=dev)
            o_strides = (n * hq * dh, hq * dh, dh)
        else:
            if out.shape != shape or out.dtype != dtype or out.device != dev:
                raise ValueError("out must have the shape, type and device of q")
            o_strides = out.stride()
            if o_strides[3] != 1:
                raise ValueError("heads must be contiguous")
            if out.requires_grad:
                refuse_autograd("out")
        if batch == 0:
            return out
        if self.pages == 0:
            raise ValueError("the cache has no pages")
        need = _workspace_bytes(self.heads, self.page, dh, self._c.format, _DTYPES[dtype], batch, n, hq, cols)
        ws = 0
        if need:
            if workspace is None or workspace.numel() < need:
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
            elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
                raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
            ws = workspace.data_ptr()
        p = sn_attend(_DTYPES[dtype], batch, n, hq, cols, dh ** -0.5 if scale is None else scale, *q_strides[:3],
                      *o_strides[:3], table_ld, mask_batch)
        on_stream_of(dev, spectral_cache_attend, self._c, p, q.data_ptr(), table.data_ptr(), lengths.data_ptr(), masks,
                     out.data_ptr(), ws, need)
        return out
