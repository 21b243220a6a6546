"""Paged caches (include/mbp.h): keys and values of many sequences in pages of 16-bit or
MXFP4 values, appending rotated rows to them, reading rows back, and attention over them.

Argument marshalling only.  Every call enqueues its work on the current stream of the
cache's device and waits for nothing; tensors that another stream produced or will use
are the caller's to order, as with any operation of PyTorch.
"""
from __future__ import annotations

import ctypes
import math

__all__ = ["PagedCache", "PagedRows", "rope_table"]


class _Cache(ctypes.Structure):
    """Mirror of mbp_paged_cache."""
    _fields_ = [("dtype", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("d_head", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p),
                ("d_pages", ctypes.c_void_p)]


class _Rows(ctypes.Structure):
    """Mirror of mbp_paged_rows."""
    _fields_ = [("n_rows", ctypes.c_int32), ("max_rows", ctypes.c_int32), ("max_slots", ctypes.c_int32),
                ("d_row_start", ctypes.c_void_p), ("d_first_slot", ctypes.c_void_p)]


class _Heads(ctypes.Structure):
    """Mirror of mbp_paged_heads."""
    _fields_ = [("d", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


_F32, _BF16, _F16, _MXFP4 = 0, 1, 2, 3  # mbp_dtype


def declare(L):
    """Argument types of the library's paged entry points."""
    P, I = ctypes.c_void_p, ctypes.c_int32
    L.mbp_paged_error.argtypes, L.mbp_paged_error.restype = [], ctypes.c_char_p
    L.mbp_paged_pool_bytes.argtypes, L.mbp_paged_pool_bytes.restype = [P], ctypes.c_size_t
    L.mbp_rope_table.argtypes, L.mbp_rope_table.restype = [P, I, I, ctypes.c_float, P], ctypes.c_int
    L.mbp_paged_append.argtypes, L.mbp_paged_append.restype = [P, P, I, P, P, P, P, P, P, I, P], ctypes.c_int
    L.mbp_paged_read.argtypes, L.mbp_paged_read.restype = [P, P, P, P, P], ctypes.c_int
    L.mbp_paged_workspace_bytes.argtypes, L.mbp_paged_workspace_bytes.restype = [P, P, I], ctypes.c_size_t
    L.mbp_paged_attend.argtypes = [P, P, I, P, P, P, P, ctypes.c_float, P, ctypes.c_size_t, P]
    L.mbp_paged_attend.restype = ctypes.c_int


def _ints(torch, name, t, device, n=None):
    """Checks an int32 tensor that the library reads in place; returns its address."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.get_device() != device.index or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 tensor on {device} is needed")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name}: {n} elements are needed, got {t.numel()}")
    return t.data_ptr()


class PagedRows:
    """The token rows of one call (mbp_paged_rows).

    ``row_start`` int32 [n_seqs + 1] and ``first_slot`` int32 [n_seqs] on the device;
    ``n_rows`` rows in the arrays that go with it; ``max_rows`` at least the most rows of one
    sequence, ``max_slots`` about the most slots that a row sees.  The two tensors are read
    by the device when a call runs, so a captured graph sees what they hold at its replay;
    the three numbers are fixed at capture.
    """

    def __init__(self, row_start, first_slot, n_rows, max_rows, max_slots):
        import torch

        self.device = row_start.device
        if self.device.type != "cuda":
            raise ValueError("row_start: a device tensor is needed")
        if first_slot.dim() != 1:
            raise ValueError("first_slot: one dimension is needed")
        self.n_seqs, self.n_rows = first_slot.numel(), int(n_rows)
        a = _ints(torch, "row_start", row_start, self.device, self.n_seqs + 1)
        b = _ints(torch, "first_slot", first_slot, self.device)
        for name, x in (("n_rows", n_rows), ("max_rows", max_rows), ("max_slots", max_slots)):
            if not 0 <= int(x) < 1 << 31:
                raise ValueError(f"{name} must be in [0, 2^31)")
        self.row_start, self.first_slot = row_start, first_slot  # kept alive
        self._c = _Rows(self.n_rows, int(max_rows), int(max_slots), a, b)
        self._ref = ctypes.addressof(self._c)


def rope_table(n_pos, d_head, base, device="cuda"):
    """Cosines and sines of rotary positions (mbp_rope_table): float32 [n_pos, d_head / 2, 2]."""
    import torch

    from . import MbpError, lib

    L = lib()
    t = torch.empty((int(n_pos), int(d_head) // 2, 2), dtype=torch.float32, device=device)
    with torch.cuda.device(t.device):
        rc = L.mbp_rope_table(t.data_ptr() or None, int(n_pos), int(d_head), float(base), torch.cuda.current_stream(t.device).cuda_stream)
    if rc:
        raise MbpError(rc, L.mbp_paged_error().decode())
    return t


class PagedCache:
    """Keys and values of ``pages.shape[0]`` sequences in pages (mbp_paged_cache).

    ``dtype`` BF16, F16 or MXFP4; ``pages`` int32 [n_seqs, max_pages] on the device, the
    caller's page table, read at every call.  The pools are allocated for ``n_pages`` pages
    (their contents undefined), or given as ``k`` and ``v``: [n_pages, n_kv_heads, page_size,
    d_head] of the 16-bit type, or uint8 [n_pages, n_kv_heads, page_size * (d_head / 2 +
    d_head / 32)] for MXFP4.
    """

    def __init__(self, dtype, n_kv_heads, d_head, page_size, *, pages, n_pages=None, k=None, v=None):
        import torch

        from . import EINVAL, MbpError, lib

        self.torch, self.L, self.error = torch, lib(), MbpError
        self.device = pages.device
        if self.device.type != "cuda" or self.device.index is None:
            raise ValueError("pages: a device tensor is needed")
        if pages.dim() != 2:
            raise ValueError("pages: int32 [n_seqs, max_pages] is needed")
        table = _ints(torch, "pages", pages, self.device)
        self.dtype, self.n_kv_heads, self.d_head, self.page_size = int(dtype), int(n_kv_heads), int(d_head), int(page_size)
        if (k is None) != (v is None) or (k is None) == (n_pages is None):
            raise ValueError("either n_pages or both pools are needed")
        self.n_pages = int(n_pages if k is None else k.shape[0])
        self._c = _Cache(self.dtype, self.n_kv_heads, self.d_head, self.page_size, self.n_pages, pages.shape[0], pages.shape[1],
                         None, None, table)
        self._ref = ctypes.addressof(self._c)
        if self.L.mbp_paged_pool_bytes(self._ref) == 0:
            raise MbpError(EINVAL, self.L.mbp_paged_error().decode())
        fp4 = self.dtype == _MXFP4
        kind = torch.uint8 if fp4 else torch.bfloat16 if self.dtype == _BF16 else torch.float16
        page = (self.page_size * (self.d_head // 2 + self.d_head // 32),) if fp4 else (self.page_size, self.d_head)
        shape = (self.n_pages, self.n_kv_heads, *page)
        if k is None:
            k, v = (torch.empty(shape, dtype=kind, device=self.device) for _ in range(2))
        for name, t in (("k", k), ("v", v)):
            if t.dtype is not kind or tuple(t.shape) != shape or t.device != self.device or not t.is_contiguous():
                raise ValueError(f"{name}: a contiguous {kind} tensor {list(shape)} on {self.device} is needed")
        self.k, self.v, self.pages, self.n_seqs = k, v, pages, pages.shape[0]
        self._c.d_k, self._c.d_v = k.data_ptr(), v.data_ptr()
        self._index = self.device.index
        self._numbers = {torch.float32: _F32, torch.bfloat16: _BF16, torch.float16: _F16}
        # the stream's address without a Stream object around it, which costs more than a launch
        self._stream = torch._C._cuda_getCurrentRawStream
        self._single = torch.cuda.device_count() == 1

    def _heads(self, name, t, n_rows, heads=None):
        shape = t.shape
        if len(shape) != 3 or shape[0] != n_rows or shape[2] != self.d_head or (heads is not None and shape[1] != heads):
            raise ValueError(f"{name}: [{n_rows}, {'heads' if heads is None else heads}, {self.d_head}] is needed, got {list(shape)}")
        if t.get_device() != self._index:
            raise ValueError(f"{name} is on {t.device}, the cache on {self.device}")
        if t.requires_grad and self.torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient: these operators have none (detach it, or use no_grad)")
        rs, hs, es = t.stride()
        if es != 1:
            raise ValueError(f"{name}: the channels of a head must be adjacent")
        number = self._numbers.get(t.dtype)
        if number is None:
            raise ValueError(f"{name}: float32, bfloat16 or float16 is needed, got {t.dtype}")
        # a tensor without elements has no address: one that is never followed stands in
        return _Heads(t.data_ptr() or 16, number, rs, hs)

    def _check_rows(self, rows):
        if rows.n_seqs != self.n_seqs or rows.device != self.device:
            raise ValueError(f"rows of {rows.n_seqs} sequences on {rows.device}, a cache of {self.n_seqs} on {self.device}")

    def _run(self, fn, *args):
        """The call on the cache's device and its current stream."""
        stream = self._stream(self._index)
        if self._single or self.torch.cuda.current_device() == self._index:
            rc = fn(*args, stream)
        else:
            with self.torch.cuda.device(self.device):
                rc = fn(*args, stream)
        if rc:
            raise self.error(rc, self.L.mbp_paged_error().decode())

    def append(self, rows, k, v, q=None, q_out=None, pos=None, rope=None):
        """Stores rows ``k``, ``v`` [n_rows, n_kv_heads, d_head] in their slots, keys rotated
        by ``rope`` (rope_table) at ``pos`` int32 [n_rows], by default the rows' slots.  With
        ``q`` [n_rows, heads, d_head] also rotates the queries, into ``q_out`` (allocated by
        default, may be ``q``), and returns them."""
        self._check_rows(rows)
        n, torch = rows.n_rows, self.torch
        ks, vs = self._heads("k", k, n, self.n_kv_heads), self._heads("v", v, n, self.n_kv_heads)
        qs = qo = None
        heads = 0
        if q is not None:
            heads = q.shape[1] if q.dim() == 3 else 0
            qs = self._heads("q", q, n)
            if q_out is None:
                q_out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
            qo = self._heads("q_out", q_out, n, heads)
        elif q_out is not None:
            raise ValueError("q_out is given without q")
        table, n_pos = None, 0
        if rope is not None:
            if rope.dtype is not torch.float32 or rope.device != self.device or not rope.is_contiguous() or rope.dim() != 3 or \
                    tuple(rope.shape[1:]) != (self.d_head // 2, 2):
                raise ValueError(f"rope: a contiguous float32 tensor [n_pos, {self.d_head // 2}, 2] on {self.device} is needed")
            table, n_pos = rope.data_ptr(), rope.shape[0]
        at = _ints(torch, "pos", pos, self.device, n)
        self._run(self.L.mbp_paged_append, self._ref, rows._ref, heads, qs and ctypes.byref(qs), qo and ctypes.byref(qo),
                  ctypes.byref(ks), ctypes.byref(vs), at, table, n_pos)
        return q_out

    def read(self, rows, dtype=None, k=None, v=None):
        """The values in the rows' slots, as two [n_rows, n_kv_heads, d_head] tensors of
        ``dtype`` (float32 by default) or in ``k`` and ``v``."""
        self._check_rows(rows)
        torch = self.torch
        shape = (rows.n_rows, self.n_kv_heads, self.d_head)
        k, v = (torch.empty(shape, dtype=dtype or torch.float32, device=self.device) if t is None else t for t in (k, v))
        ks, vs = self._heads("k", k, rows.n_rows, self.n_kv_heads), self._heads("v", v, rows.n_rows, self.n_kv_heads)
        self._run(self.L.mbp_paged_read, self._ref, rows._ref, ctypes.byref(ks), ctypes.byref(vs))
        return k, v

    def attend(self, rows, q, out=None, lo=None, hi=None, scale=None):
        """Attention of ``q`` [n_rows, heads, d_head] over slots ``lo`` .. ``hi`` - 1 (int32
        [n_rows]; by default 0 and the row's own slot + 1) of each row's sequence.  Rows that
        belong to no sequence are 0 in an allocated ``out`` and left alone in a given one,
        which may be ``q``."""
        self._check_rows(rows)
        n, torch = rows.n_rows, self.torch
        qs = self._heads("q", q, n)
        heads = q.shape[1]
        if out is None:
            out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        os_ = self._heads("out", out, n, heads)
        low, high = _ints(torch, "lo", lo, self.device, n), _ints(torch, "hi", hi, self.device, n)
        need = self.L.mbp_paged_workspace_bytes(self._ref, rows._ref, heads)
        # allocated for each call: the caching allocator keeps it with the stream, or with
        # the graph under capture, so that no two of them share it
        work = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        self._run(self.L.mbp_paged_attend, self._ref, rows._ref, heads, ctypes.byref(qs), ctypes.byref(os_), low, high,
                  1.0 / math.sqrt(self.d_head) if scale is None else float(scale), work.data_ptr() if need else None, need)
        return out
