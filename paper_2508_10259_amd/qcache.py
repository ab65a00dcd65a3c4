"""The 8-bit K/V cache of one layer over the C ABI (ams_qcache_append, ams_qcache_attend).

``QuantCache`` binds the cache's device tensors; ``append`` writes new tokens, ``attend`` and
``attend_selected`` run the causal attention of their queries.  Lengths and offsets are device
tensors that the calls read on the device, so a decode step can be captured into a graph and
replayed.  Everything runs on torch's current stream.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Tuple

import torch

from . import capi

PAGE = 64
E4M3 = torch.float8_e4m3fn
_DTYPES = {torch.float32: capi.AMS_F32, torch.bfloat16: capi.AMS_BF16, torch.float16: capi.AMS_F16}


def _raw_stream(index: int) -> int:
    return torch._C._cuda_getCurrentRawStream(index)


def _want(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


class QuantCache:
    """Pools, scales, bounds and page table of one layer (layouts as in ``include/ams.h``).

    k [pages, heads, 64, dim] and v [pages, heads, 16, dim, 4] float8_e4m3fn; k_scale, v_scale
    [pages, heads] float32; k_bounds [pages, heads, 2, dim] int8; page_table [rows, pages per row]
    int32 (entries outside the pool hold no positions).  All contiguous on one device,
    which is the current one at every call.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                 k_bounds: torch.Tensor, page_table: torch.Tensor):
        _want(k.dim() == 4 and k.shape[2] == PAGE, "k must be [pages, heads, 64, head_dim]")
        pages, heads, _, dim = k.shape
        for t, name, shape, dtype in (
                (k, "k", (pages, heads, PAGE, dim), E4M3), (v, "v", (pages, heads, PAGE // 4, dim, 4), E4M3),
                (k_scale, "k_scale", (pages, heads), torch.float32),
                (v_scale, "v_scale", (pages, heads), torch.float32),
                (k_bounds, "k_bounds", (pages, heads, 2, dim), torch.int8),
                (page_table, "page_table", tuple(page_table.shape), torch.int32)):
            _want(tuple(t.shape) == shape and t.dtype == dtype and t.is_contiguous() and t.device == k.device,
                  f"{name} must be a contiguous {dtype} tensor of shape {shape} on {k.device}")
        _want(page_table.dim() == 2, "page_table must be [rows, pages_per_row]")
        self.lib = lib = capi.load()
        self.k, self.v, self.k_scale, self.v_scale, self.k_bounds = k, v, k_scale, v_scale, k_bounds
        self.page_table = page_table
        self.n_kv_heads, self.head_dim, self.rows = heads, dim, page_table.shape[0]
        self.device = k.device
        self.c = capi.QCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), k_bounds.data_ptr(),
                             page_table.data_ptr(), pages, heads, dim, self.rows, page_table.shape[1])
        # (a decode step makes these calls for every layer, so what does not change is kept)
        self._ref = C.byref(self.c)
        self._append, self._attend, self._workspace = \
            lib.ams_qcache_append, lib.ams_qcache_attend, lib.ams_qcache_workspace_bytes
        self._index = 0 if k.device.index is None else k.device.index
        self._off_shape, self._len_shape = torch.Size((self.rows + 1,)), torch.Size((self.rows,))

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_table: torch.Tensor) -> "QuantCache":
        """New pools of n_pages pages on page_table's device (every code, scale and bound zero)."""
        dev = page_table.device
        return cls(torch.zeros(n_pages, n_kv_heads, PAGE, head_dim, dtype=torch.uint8, device=dev).view(E4M3),
                   torch.zeros(n_pages, n_kv_heads, PAGE // 4, head_dim, 4, dtype=torch.uint8, device=dev).view(E4M3),
                   torch.zeros(n_pages, n_kv_heads, device=dev), torch.zeros(n_pages, n_kv_heads, device=dev),
                   torch.zeros(n_pages, n_kv_heads, 2, head_dim, dtype=torch.int8, device=dev), page_table)

    def _rows(self, tok_off: torch.Tensor, lens: torch.Tensor) -> None:
        if tok_off.dtype != torch.int32 or tok_off.shape != self._off_shape or not tok_off.is_contiguous() \
                or tok_off.device != self.device:
            raise ValueError("tok_off must be a contiguous int32 tensor [rows + 1] of the cache's device")
        if lens.dtype != torch.int32 or lens.shape != self._len_shape or not lens.is_contiguous() \
                or lens.device != self.device:
            raise ValueError("lens must be a contiguous int32 tensor [rows] of the cache's device")

    def _tensor(self, t: torch.Tensor, name: str) -> int:
        """Token stride of a [n_tok, heads, head_dim] tensor whose heads lie one after another."""
        shape, stride, dim = t.shape, t.stride(), self.head_dim
        if len(shape) != 3 or shape[2] != dim or t.dtype not in _DTYPES or t.device != self.device:
            raise ValueError(f"{name} must be a float32, bfloat16 or float16 tensor [n_tok, heads, {dim}] of the cache's "
                             "device")
        n, heads, _ = shape
        if n * heads and (stride[2] != 1 or (heads > 1 and stride[1] != dim)):
            raise ValueError(f"{name}: the heads of a token must lie one after another")
        return stride[0] if n > 1 else heads * dim

    def append(self, k: torch.Tensor, v: torch.Tensor, tok_off: torch.Tensor, lens: torch.Tensor, *,
               max_new: Optional[int] = None) -> None:
        """Stores the tokens' keys and values [n_tok, heads, head_dim]: row b's are tokens tok_off[b] ..
        tok_off[b + 1] - 1, its last one at position lens[b] - 1.  max_new: at least the most tokens of a row
        (default n_tok)."""
        self._rows(tok_off, lens)
        ldk, ldv = self._tensor(k, "k"), self._tensor(v, "v")
        n = k.shape[0]
        if k.shape != v.shape or k.shape[1] != self.n_kv_heads or k.dtype != v.dtype:
            raise ValueError("k and v must have the cache's heads, one shape and one type")
        status = self._append(self._ref, tok_off.data_ptr(), lens.data_ptr(), n, max(n, 1) if max_new is None else max_new,
                              k.data_ptr(), ldk, v.data_ptr(), ldv, _DTYPES[k.dtype], _raw_stream(self._index))
        if status:
            capi.check(status, "ams_qcache_append")

    def attend(self, q: torch.Tensor, tok_off: torch.Tensor, lens: torch.Tensor, *, max_new: Optional[int] = None,
               max_len: Optional[int] = None, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Causal attention of the tokens' queries [n_tok, n_heads, head_dim] over everything their rows hold.
        max_new: at least the most tokens of a row.  It chooses the kernel, and the default, n_tok, takes them for one
        row's: name it where there are several rows (64 rows of one token, 200 to 768 positions: 58 us with max_new=1, 68 to 73
        without).  max_len: about the longest row (default: the capacity); scale: default 1 / sqrt(head_dim)."""
        return self._run(q, tok_off, lens, 0, max_new, max_len, scale, out, None)

    def attend_selected(self, q: torch.Tensor, tok_off: torch.Tensor, lens: torch.Tensor, n_select: int, *,
                        max_new: Optional[int] = None, max_len: Optional[int] = None, scale: Optional[float] = None,
                        out: Optional[torch.Tensor] = None,
                        selected: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The same over n_select pages of each token and KV head.  Returns (out, selected): the chosen
        pages of the row [n_tok, kv heads, n_select] int32, increasing, then -1."""
        if n_select < 1:
            raise ValueError("n_select must be >= 1")
        if selected is None:
            selected = torch.empty((q.shape[0], self.n_kv_heads, n_select), dtype=torch.int32, device=self.device)
        elif selected.dtype != torch.int32 or not selected.is_contiguous() or selected.device != self.device \
                or tuple(selected.shape) != (q.shape[0], self.n_kv_heads, n_select):
            raise ValueError("selected must be a contiguous int32 tensor [n_tok, kv heads, n_select] of the cache's device")
        return self._run(q, tok_off, lens, n_select, max_new, max_len, scale, out, selected), selected

    def _run(self, q, tok_off, lens, n_select, max_new, max_len, scale, out, selected):
        self._rows(tok_off, lens)
        ldq = self._tensor(q, "q")
        n, heads, dim = q.shape
        if out is None:
            out = torch.empty((n, heads, dim), dtype=q.dtype, device=self.device)
            ldo = heads * dim
        else:
            ldo = self._tensor(out, "out")
            if out.shape != q.shape or out.dtype != q.dtype:
                raise ValueError("out must have q's shape and type")
        if max_new is None:
            max_new = max(n, 1)
        if max_len is None:
            max_len = self.c.pages_per_row * PAGE
        ws, need = None, self._workspace(self._ref, heads, n, max_new, max_len, n_select)
        if need and selected is not None:
            need -= 4 * selected.numel()  # (the size counts a list of the pages chosen, which has a place of its own here)
        if need > 1:
            # from the allocator at every call: its memory follows the stream, and a captured graph's stays with it
            ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        status = self._attend(
            self._ref, tok_off.data_ptr(), lens.data_ptr(), n, max_new, max_len, heads, q.data_ptr(), ldq, out.data_ptr(),
            ldo, _DTYPES[q.dtype], 1 / math.sqrt(dim) if scale is None else scale, n_select,
            None if selected is None else selected.data_ptr(), None if ws is None else ws.data_ptr(), need,
            _raw_stream(self._index))
        if status:
            capi.check(status, "ams_qcache_attend")
        return out
