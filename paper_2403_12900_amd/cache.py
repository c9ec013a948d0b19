"""The 4-bit KV cache's operators on torch tensors: a thin binding of spr_cache_rotary, spr_cache_append, spr_cache_read,
spr_cache_attention, spr_cache_fork and spr_cache_move.

Argument marshalling only, as in tree.py: shapes, types and devices are checked here, all other checks are the library's.
Inference only: tensors that want gradients or carry tangents are refused.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Union

import numpy as np
import torch

from .binding import SPR_OK, SprCacheBatch, SprKv4View, SprPages, SprRotary, _check, _ptr, load_library
from .tree import _DTYPES, KVView, OpHandle, _int32, _refuse


class KV4View:
    """A paged KV cache in 4 bits (spr_kv4_view): data [layers, blocks, KV heads, 17 * head_dim] bytes in the tile order that
    the header gives, and the int32 block table [slots, blocks per slot], contiguous on one device.  A fresh cache may hold
    anything: no operator reads positions that were not appended."""

    def __init__(self, data: torch.Tensor, block_table: torch.Tensor):
        if data.dim() != 4 or data.dtype != torch.uint8 or data.shape[3] % 17:
            _refuse("kv4 view: data must be uint8 [layers, blocks, kv_heads, 17 * head_dim]")
        if block_table.dim() != 2 or block_table.dtype != torch.int32:
            _refuse("kv4 view: the block table must be int32 [slots, blocks per slot]")
        if not (data.is_contiguous() and block_table.is_contiguous()):
            _refuse("kv4 view: data and the block table must be contiguous")
        if block_table.device != data.device:
            _refuse("kv4 view: data and the block table must be on one device")
        self.data, self.block_table, self.index = data, block_table, data.get_device()
        self.head_dim = data.shape[3] // 17
        self.n_kv_heads = data.shape[2]
        self._c = SprKv4View(data.data_ptr(), data.shape[0], data.shape[1], data.shape[2], self.head_dim,
                             block_table.data_ptr(), block_table.shape[0], block_table.shape[1])
        self.ref = ctypes.byref(self._c)

    @staticmethod
    def empty(layers: int, blocks: int, n_kv_heads: int, head_dim: int, slots: int, blocks_per_slot: int, device=0) -> "KV4View":
        """A cache of its own, with a table of zeros."""
        return KV4View(torch.empty(layers, blocks, n_kv_heads, 17 * head_dim, dtype=torch.uint8, device=device),
                       torch.zeros(slots, blocks_per_slot, dtype=torch.int32, device=device))


class CacheBatch:
    """The requests of one call (spr_cache_batch): per request its slot, the positions before its rows, and its rows."""

    def __init__(self, slots: Sequence[int], lens: Sequence[int], rows: Sequence[int]):
        # Copies: what the library reads later stays as it was checked here.
        self._a = [_int32(x, name, "cache batch") for x, name in ((slots, "slots"), (lens, "lens"), (rows, "rows"))]
        n = len(self._a[0])
        if any(len(x) != n for x in self._a):
            _refuse("cache batch: slots, lens and rows must be of one length")
        self.n, self.rows = n, int(np.maximum(self._a[2], 0).sum(dtype=np.int64))
        self._c = SprCacheBatch(n, *(_ptr(x) for x in self._a))
        self.ref = ctypes.byref(self._c)


class Rotary:
    """Rotary positions (spr_rotary_init): the first dims dimensions of a head, in pairs (d, d + dims / 2) (layout "half") or
    (2d, 2d + 1) ("pairs"), turned at base^(-2k / dims); factor > 1 lowers the frequencies that turn seldom over the
    original length, and amplitude scales what is turned."""

    def __init__(self, dims: int, layout: str = "half", base: float = 10000.0, factor: float = 1.0, original: float = 0.0,
                 low: float = 1.0, high: float = 32.0, amplitude: float = 1.0):
        if layout not in ("half", "pairs"):
            _refuse('rotary: layout must be "half" or "pairs"')
        self._c = SprRotary()
        self.ref = ctypes.byref(self._c)
        _check(load_library().spr_rotary_init(dims, layout == "pairs", base, factor, original, low, high, amplitude, self.ref))
        self.dims, self.layout = dims, layout


class CacheOps(OpHandle):
    """The 4-bit cache's operators of one device (spr_cache_ops_init)."""

    _prefix = "spr_cache_ops"

    def rotary(self, rotary: Rotary, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None):
        """Rotary positions (spr_cache_rotary): x [rows, heads, head_dim], fp32 or bf16, rows at any stride, positions int32
        [rows]; returns out like it (which may be x itself)."""
        dtype = _DTYPES.get(x.dtype)
        if x.dim() != 3 or dtype is None:
            _refuse("cache rotary: x must be [rows, heads, head_dim], fp32 or bf16")
        self._no_grad("cache rotary", x, x if out is None else out)
        rows, heads, hd = x.shape
        p_positions = self._vector("cache rotary: positions", positions, torch.int32, rows)
        xs = self._row_stride("cache rotary", x, heads, hd)
        out, os = self._out("cache rotary", x, out, heads, hd)
        self._enter()
        self._done(self.lib.spr_cache_rotary(self.h, rotary.ref, rows, heads, hd, dtype, p_positions, x.data_ptr(), xs,
                                             out.data_ptr(), os))
        return out

    def append(self, kv: KV4View, layer: int, batch: CacheBatch, k: torch.Tensor, v: torch.Tensor, rotary: Optional[Rotary] = None):
        """Writes the rows' keys and values (spr_cache_append): k and v [rows, KV heads, head_dim], fp32 or bf16, rows at any
        stride; keys are turned at their cache positions first where rotary is given."""
        shape, dtype = (batch.rows, kv.n_kv_heads, kv.head_dim), _DTYPES.get(k.dtype)
        if k.shape != shape or v.shape != shape or dtype is None or v.dtype != k.dtype:
            _refuse("cache append: k and v must be [rows, kv_heads, head_dim] of one type, fp32 or bf16")
        self._no_grad("cache append", k, v)
        ks = self._row_stride("cache append", k, shape[1], shape[2])
        vs = self._row_stride("cache append", v, shape[1], shape[2])
        self._same_device("cache append", kv)
        self._enter()
        self._done(self.lib.spr_cache_append(self.h, kv.ref, layer, batch.ref, None if rotary is None else rotary.ref, dtype,
                                             k.data_ptr(), ks, v.data_ptr(), vs))

    def read(self, kv: KV4View, layer: int, batch: CacheBatch, dtype: torch.dtype = torch.float32):
        """The values that the cache holds at the rows (spr_cache_read): k and v [rows, KV heads, head_dim]."""
        code = _DTYPES.get(dtype)
        if code is None:
            _refuse("cache read: dtype must be fp32 or bf16")
        self._same_device("cache read", kv)
        heads, hd = kv.n_kv_heads, kv.head_dim
        k = torch.empty(batch.rows, heads, hd, dtype=dtype, device=kv.data.device)
        v = torch.empty_like(k)
        self._enter()
        self._done(self.lib.spr_cache_read(self.h, kv.ref, layer, batch.ref, code, k.data_ptr(), heads * hd, v.data_ptr(),
                                           heads * hd))
        return k, v

    def attention(self, kv: KV4View, layer: int, batch: CacheBatch, q: torch.Tensor, out: Optional[torch.Tensor] = None):
        """Attention of the rows over the cache (spr_cache_attention): q [rows, heads, head_dim], fp32 or bf16, rows at any
        stride; returns out like it."""
        hd, dtype = kv.head_dim, _DTYPES.get(q.dtype)
        if q.dim() != 3 or q.shape[0] != batch.rows or q.shape[2] != hd or dtype is None:
            _refuse("cache attention: q must be [rows, heads, head_dim], fp32 or bf16")
        self._no_grad("cache attention", q, q if out is None else out)
        heads = q.shape[1]
        qs = self._row_stride("cache attention", q, heads, hd)
        out, os = self._out("cache attention", q, out, heads, hd)
        self._same_device("cache attention", kv)
        self._enter()
        self._done(self.lib.spr_cache_attention(self.h, kv.ref, layer, batch.ref, heads, dtype, q.data_ptr(), qs,
                                                out.data_ptr(), os))
        return out

    def fork(self, kv: Union[KV4View, KVView], source: Sequence[int], target: Sequence[int], lens: Sequence[int],
             fresh: Sequence[int]):
        """Forks requests (spr_cache_fork): slot target[i] continues the first lens[i] positions of slot source[i], whose full
        blocks it shares; fresh[i] takes a copy of the last, partly filled one.  Any paged cache."""
        n, at = self._lists("cache fork", source=source, target=target, lens=lens, fresh=fresh)
        pages = self._pages("cache fork", kv)
        self._enter()
        self._done(self.lib.spr_cache_fork(self.h, pages, n, at, at + 4 * n, at + 8 * n, at + 12 * n))

    def move(self, kv: Union[KV4View, KVView], src: Sequence[int], dst: Sequence[int]):
        """Moves blocks src[i] to dst[i] in every layer, and the table's entries with them (spr_cache_move).  Any paged cache."""
        n, at = self._lists("cache move", src=src, dst=dst)
        pages = self._pages("cache move", kv)
        self._enter()
        self._done(self.lib.spr_cache_move(self.h, pages, n, at, at + 4 * n))

    _staged: Optional[np.ndarray] = None  # a call's lists, one after the other

    def _lists(self, what, **lists):
        """The lists' common length, and the address at which they stand one after the other for the call."""
        a = [x if type(x) is np.ndarray and x.dtype == np.int32 and x.ndim == 1 else _int32(x, name, what)
             for name, x in lists.items()]
        n = len(a[0])
        for x in a:
            if len(x) != n:
                _refuse(f"{what}: {', '.join(lists)} must be of one length")
        if self._staged is None or len(self._staged) < n * len(a):
            self._staged = np.empty(max(512, n * len(a)), dtype=np.int32)
            self._staged_at = self._staged.ctypes.data
        for i, x in enumerate(a):
            self._staged[i * n:(i + 1) * n] = x
        return n, self._staged_at

    def _pages(self, what, kv):
        self._same_device(what, kv)
        if not isinstance(kv, KV4View):
            self._no_grad(what, kv.k, kv.v)
            if kv.of_model:
                _refuse(f"{what}: a model's own cache: its slots own its blocks")
        ref = getattr(kv, "_pages", None)
        if ref is None:  # as lasting as the view's own record
            k, v = (kv.data, None) if isinstance(kv, KV4View) else (kv.k, kv.v)
            layers, blocks, heads, tile = k.shape
            ref = kv._pages = ctypes.byref(SprPages(k.data_ptr(), None if v is None else v.data_ptr(),
                                                    heads * tile * k.element_size(), layers, blocks, kv.block_table.data_ptr(),
                                                    *kv.block_table.shape))
        return ref

    def _done(self, status):
        if status != SPR_OK:
            _check(status)

    def _same_device(self, what, kv):
        if kv.index != self.index:
            _refuse(f"{what}: the cache must be on {self.device}")

    def _out(self, what, x, out, heads, hd):
        """The output, a new one like x if none is given, and its row stride."""
        if out is None:
            return torch.empty_like(x, memory_format=torch.contiguous_format), heads * hd
        if out.shape != x.shape or out.dtype != x.dtype:
            _refuse(f"{what}: out must be like its input")
        return out, self._row_stride(what, out, heads, hd)

    def _row_stride(self, what, t, heads, hd):
        row, head, one = t.stride()
        if t.get_device() != self.index or one != 1 or (heads > 1 and head != hd):
            _refuse(f"{what}: its tensors must be on {self.device} with contiguous rows")
        return row if t.shape[0] > 1 else heads * hd  # a single row's stride does not matter
