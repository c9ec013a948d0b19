"""Drafted-tree operators on torch tensors: a thin binding of spr_tree_attention, spr_tree_verify and spr_tree_keep.

Argument marshalling only, as in binding.py: shapes, types and devices are checked here (the C ABI sees pointers), all
other checks are the library's.  PyTorch provides device memory and the stream: each call runs on the device's current
stream.
"""
from __future__ import annotations

import ctypes
from array import array
from typing import Optional, Sequence

import numpy as np
import torch
from torch.autograd import forward_ad

from .binding import (KV_BLOCK, SPR_BF16, SPR_ERR_INVALID_ARG, SPR_F32, SproutError, SprKvView, SprTreeBatch, _check, _ptr,
                      load_library)

_DTYPES = {torch.float32: SPR_F32, torch.bfloat16: SPR_BF16}


def _refuse(msg: str):
    raise SproutError(SPR_ERR_INVALID_ARG, msg)


def _int32(x, name, what="tree batch"):
    """x as a vector of int32 of its own, each entry with its value."""
    if type(x) is np.ndarray and x.dtype == np.int32 and x.ndim == 1:
        return x.copy()
    try:
        if isinstance(x, (list, tuple)) and len(x):
            return np.frombuffer(array("i", x), dtype=np.int32)  # whole numbers of any type; OverflowError past 32 bits
    except OverflowError:
        _refuse(f"{what}: {name} must be whole numbers of 32 bits")
    except TypeError:
        pass  # floats, for one
    try:
        a = np.array(x.tolist() if isinstance(x, torch.Tensor) else x).reshape(-1)
        if a.dtype.kind == "O":
            return np.frombuffer(array("i", a.tolist()), dtype=np.int32)
        if a.size == 0 or a.dtype.kind in "biu" or a.dtype.kind == "f" and (np.abs(a) < 2 ** 31).all():
            b = a.astype(np.int32)
            if (a == b).all():
                return b
    except (TypeError, ValueError, OverflowError):
        pass
    _refuse(f"{what}: {name} must be whole numbers of 32 bits")


class KVView:
    """A paged KV cache (spr_kv_view): k and v [layers, blocks, KV heads, 16 * head_dim] in the tile order that the header
    gives, fp32 or bf16, and the int32 block table [slots, blocks per slot], all contiguous on one device."""

    of_model = False  # a model's own cache, whose slots own its blocks

    def __init__(self, k: torch.Tensor, v: torch.Tensor, block_table: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype not in _DTYPES or v.dtype != k.dtype:
            _refuse("kv view: k and v must be [layers, blocks, kv_heads, 16 * head_dim] of one type, fp32 or bf16")
        if k.shape[3] % KV_BLOCK or block_table.dim() != 2 or block_table.dtype != torch.int32:
            _refuse("kv view: blocks hold 16 positions, and the block table is int32 [slots, blocks per slot]")
        if not (k.is_contiguous() and v.is_contiguous() and block_table.is_contiguous()):
            _refuse("kv view: k, v and the block table must be contiguous")
        if v.device != k.device or block_table.device != k.device:
            _refuse("kv view: k, v and the block table must be on one device")
        self.k, self.v, self.block_table, self.index = k, v, block_table, k.get_device()
        self.head_dim = k.shape[3] // KV_BLOCK
        self.n_kv_heads = k.shape[2]
        self._c = SprKvView(k.data_ptr(), v.data_ptr(), _DTYPES[k.dtype], k.shape[0], k.shape[1], k.shape[2],
                            self.head_dim, block_table.data_ptr(), block_table.shape[0], block_table.shape[1])
        self.ref = ctypes.byref(self._c)


class TreeBatch:
    """The drafted trees of one call (spr_tree_batch): per request its slot, cached positions and number of nodes, and all
    nodes' parents (-1 for a root), request after request.  slots and lens may be None for verification alone."""

    def __init__(self, slots: Optional[Sequence[int]], lens: Optional[Sequence[int]], n_nodes: Sequence[int],
                 parents: Sequence[int]):
        # Copies: what the library reads later stays as it was checked here.
        self._a = [None if x is None else _int32(x, name) for x, name in
                   ((slots, "slots"), (lens, "lens"), (n_nodes, "n_nodes"), (parents, "parents"))]
        n = len(self._a[2])
        if any(x is not None and len(x) != n for x in self._a[:2]):
            _refuse("tree batch: slots, lens and n_nodes must be of one length")
        # A negative count must not make the sum match: every entry is checked by the library, the length here.
        if len(self._a[3]) != int(np.maximum(self._a[2], 0).sum(dtype=np.int64)):
            _refuse("tree batch: parents must have sum(n_nodes) entries")
        self.n, self.rows = n, len(self._a[3])
        self._floats = ctypes.c_float * n
        self._c = SprTreeBatch(n, *(None if x is None else _ptr(x) for x in self._a))
        self.ref = ctypes.byref(self._c)

    def temperatures(self, temperature):
        """The request temperatures as the C ABI takes them (one number, or one per request; None: 1)."""
        if temperature is None:
            return None
        if not hasattr(temperature, "__len__"):
            temperature = [temperature] * self.n
        if len(temperature) != self.n:
            _refuse("tree batch: one temperature per request")
        return self._floats(*temperature)


class OpHandle:
    """An operator handle of the library on one device, in a torch workspace.

    Calls enqueue on the device's current stream; a call on another stream than the last one's first waits for that one.
    Calls that a graph captures wait for nothing and are waited for by nothing (the capture's own order holds, and the
    caller orders replays): eager calls before and after a capture wait for each other.  The handle outlives the graphs
    that hold its calls."""

    _prefix: str  # of the handle's entry points

    def __init__(self, device: int = 0):
        self.lib = load_library()
        self.index = device
        self.device = torch.device("cuda", device)
        self.ws = torch.empty(int(self._entry("workspace_bytes")()), dtype=torch.uint8, device=self.device)
        # The last eager call's stream; the handle's own (a captured call's, too), and whether they are one.
        self.stream = torch.cuda.current_stream(self.device)
        self.raw_stream, self.eager = self.stream.cuda_stream, True
        self.h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(self._entry("init")(self.ws.data_ptr(), self.ws.numel(), self.raw_stream, ctypes.byref(self.h)))

    def _entry(self, name):
        return getattr(self.lib, f"{self._prefix}_{name}")

    def _enter(self):
        """Moves the handle to the device's current stream."""
        raw = torch._C._cuda_getCurrentRawStream(self.index)
        if raw == self.raw_stream and self.eager:
            return
        s = torch.cuda.current_stream(self.device)
        with torch.cuda.device(self.device):
            self.eager = not torch.cuda.is_current_stream_capturing()
            if self.eager:
                if raw != self.stream.cuda_stream:
                    s.wait_stream(self.stream)
                    self.ws.record_stream(s)
                self.stream = s
        if raw != self.raw_stream:
            _check(self._entry("set_stream")(self.h, raw))
            self.raw_stream = raw

    def _vector(self, what, t, dtype, n):
        """Address of a contiguous vector of n elements on the handle's device."""
        if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or t.get_device() != self.index or not t.is_contiguous():
            _refuse(f"{what} must be a contiguous {dtype} tensor of {n} elements on {self.device}")
        return t.data_ptr()

    def _no_grad(self, what, *tensors):
        """Refuses what autograd would follow: tensors that want gradients, or carry a tangent."""
        if forward_ad._current_level >= 0 and any(forward_ad.unpack_dual(x).tangent is not None for x in tensors):
            _refuse(f"{what}: it has no gradient; detach its inputs, which carry a tangent")
        for x in tensors:
            if x.requires_grad and torch.is_grad_enabled():
                _refuse(f"{what}: it has no gradient; detach its inputs, or call it under torch.no_grad()")

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            self._entry("release")(self.h)
            self.h = ctypes.c_void_p()
        self.ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class TreeOps(OpHandle):
    """The drafted-tree operators of one device (spr_tree_ops_init)."""

    _prefix = "spr_tree_ops"

    def attention(self, kv: KVView, layer: int, batch: TreeBatch, q: torch.Tensor, out: Optional[torch.Tensor] = None):
        """Attention of the trees' nodes (spr_tree_attention): q [rows, heads, head_dim], fp32 or bf16, rows at any stride;
        returns out like it.  Inference only: inputs that want gradients are refused."""
        hd = kv.head_dim
        if q.dim() != 3 or q.shape[0] != batch.rows or q.shape[2] != hd or q.dtype not in _DTYPES:
            _refuse("tree attention: q must be [rows, heads, head_dim], fp32 or bf16")
        rows, heads, _ = q.shape
        self._no_grad("tree attention", q, kv.k, kv.v, q if out is None else out)
        if out is None:
            out = q.new_empty(rows, heads, hd)
        elif out.shape != q.shape or out.dtype != q.dtype:
            _refuse("tree attention: out must be like q")
        qs, os = self._row_stride(q, heads, hd), self._row_stride(out, heads, hd)
        if kv.index != self.index:
            _refuse(f"tree attention: the cache must be on {self.device}")
        self._enter()
        _check(self.lib.spr_tree_attention(self.h, kv.ref, layer, batch.ref, heads, _DTYPES[q.dtype], q.data_ptr(), qs,
                                           out.data_ptr(), os))
        return out

    def _row_stride(self, t, heads, hd):
        row, head, one = t.stride()
        if t.get_device() != self.index or one != 1 or (heads > 1 and head != hd):
            _refuse(f"tree attention: q and out must be on {self.device} with contiguous rows")
        return row if t.shape[0] > 1 else heads * hd  # a single row's stride does not matter

    def verify(self, batch: TreeBatch, tokens: torch.Tensor, logits: torch.Tensor, accept: Optional[torch.Tensor] = None,
               sample: Optional[torch.Tensor] = None, draft_probs: Optional[torch.Tensor] = None, temperature=None):
        """Verification (spr_tree_verify): tokens int32 [rows], logits [rows, vocab] (fp32 or bf16, rows at any stride),
        accept fp32 [rows] and sample fp32 [n] uniform in [0, 1), draft_probs like logits.  Returns (emitted, path) int32
        [rows] and count int32 [n]."""
        rows, n = batch.rows, batch.n
        if logits.dim() != 2 or logits.shape[0] != rows or logits.dtype not in _DTYPES:
            _refuse("tree verify: logits must be [rows, vocab], fp32 or bf16")
        vocab = logits.shape[1]
        ls = self._vocab_stride(logits, rows, vocab)
        ds, p_draft = 0, None
        if draft_probs is not None:
            if draft_probs.shape != logits.shape or draft_probs.dtype != logits.dtype:
                _refuse("tree verify: draft_probs must be like logits")
            ds, p_draft = self._vocab_stride(draft_probs, rows, vocab), draft_probs.data_ptr()
        p_tokens = self._vector("tree verify: tokens", tokens, torch.int32, rows)
        p_accept = None if accept is None else self._vector("tree verify: accept", accept, torch.float32, rows)
        p_sample = None if sample is None else self._vector("tree verify: sample", sample, torch.float32, n)
        temps = batch.temperatures(temperature)
        emitted, path, count = tokens.new_empty(2 * rows + n).split((rows, rows, n))
        self._enter()
        at = emitted.data_ptr()
        _check(self.lib.spr_tree_verify(self.h, batch.ref, vocab, _DTYPES[logits.dtype], p_tokens, logits.data_ptr(), ls,
                                        p_draft, ds, temps, p_accept, p_sample, at, at + 4 * rows, at + 8 * rows))
        return emitted, path, count

    def _vocab_stride(self, t, rows, vocab):
        row, one = t.stride()
        if t.get_device() != self.index or (vocab > 1 and one != 1):
            _refuse(f"tree verify: logits and draft_probs must be on {self.device} with contiguous rows")
        return row if rows > 1 else vocab

    def keep(self, kv: KVView, batch: TreeBatch, path: torch.Tensor, count: torch.Tensor):
        """Closes the trees in every layer of the cache (spr_tree_keep); path and count as verify returns them."""
        p_path = self._vector("tree keep: path", path, torch.int32, batch.rows)
        p_count = self._vector("tree keep: count", count, torch.int32, batch.n)
        if kv.index != self.index:
            _refuse(f"tree keep: the cache must be on {self.device}")
        self._enter()
        _check(self.lib.spr_tree_keep(self.h, kv.ref, batch.ref, p_path, p_count))
