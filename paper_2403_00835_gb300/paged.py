"""Python binding of the paged key/value cache in include/cllm_paged.h (argument
marshalling only).

A step of a serving loop over requests that come and go::

    tables = PageTables.empty(n_pages, page_size, max_batch, width)
    rows = PageRows.empty(max_batch, max_rows)
    cache = PagedCache(k_pool, v_pool, n_heads)   # pools [layer][page][head][position][hd]

    plan(tables, rows, ctx, new_rows)             # pages, slots, positions of the step
    for layer in ...:
        cache.append(layer, k, v, rows.slots, q=q, q_out=q, rope=rope, positions=rows.positions)
        cache.attention(layer, q, rows, tables, out=o)

Calls queue their work on ``stream`` (a torch stream; None: the current one) and
return; tensors are the caller's and are not copied.  Arguments of the wrong
type, device or shape raise ValueError, what the library refuses CllmError;
``PagedCache.check`` waits and raises for what only the device could see.
"""
from __future__ import annotations

import ctypes
import struct
from contextlib import nullcontext
from typing import Optional

import torch

from . import cllm as _c

CLLM_F16 = 2
DTYPES = {torch.float32: _c.CLLM_F32, torch.bfloat16: _c.CLLM_BF16, torch.float16: CLLM_F16}

# Every function declared in include/cllm_paged.h.
EXPORTS = ("cllm_page_plan", "cllm_paged_create", "cllm_paged_destroy", "cllm_paged_status", "cllm_paged_append",
           "cllm_paged_attention")


class _Tables(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("held", ctypes.c_void_p), ("ring", ctypes.c_void_p),
                ("state", ctypes.c_void_p), ("max_batch", ctypes.c_int), ("width", ctypes.c_int),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int)]


class _Rows(ctypes.Structure):
    _fields_ = [("row_start", ctypes.c_void_p), ("seq_len", ctypes.c_void_p), ("granted", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("max_rows", ctypes.c_int)]


class _Desc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int), ("layers", ctypes.c_int),
                ("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("n_kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("n_heads", ctypes.c_int), ("stride_layer", ctypes.c_int64),
                ("stride_page", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("stride_pos", ctypes.c_int64)]


# cllm_paged_rows and cllm_paged_attn as they lie in memory (native alignment): one call
# fills them, which is a third of what a ctypes structure's fields take.
_ROWS_IN = struct.Struct("@2i4P4q3Pi")
_ATTN = struct.Struct("@3i3P4q3PifiPi")

_lib = None


def load():
    """The library with this header's signatures."""
    global _lib
    if _lib is None:
        lib = _c.load()
        vp, i = ctypes.c_void_p, ctypes.c_int
        lib.cllm_page_plan.argtypes = [vp, vp, vp, i, vp, vp, vp]
        lib.cllm_paged_create.argtypes = [ctypes.POINTER(_Desc), ctypes.POINTER(vp)]
        lib.cllm_paged_destroy.argtypes = [vp]
        lib.cllm_paged_destroy.restype = None
        lib.cllm_paged_status.argtypes = [vp, vp]
        lib.cllm_paged_append.argtypes = [vp, vp, vp]
        lib.cllm_paged_attention.argtypes = [vp, vp, vp]
        for name in EXPORTS:
            if name != "cllm_paged_destroy":
                getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


def _tensor(t, what: str, dtype, shape=None, index=None):
    """A contiguous CUDA tensor's address."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()):
        raise ValueError(f"{what}: need a contiguous {dtype} CUDA tensor")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what}: need shape {tuple(shape)}, got {tuple(t.shape)}")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{what}: on {t.device}, the others on cuda:{index}")
    return t.data_ptr()


# the current stream's handle without the Stream object around it (a sixth of a call)
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream, index: int) -> int:
    if stream is None:
        return _current(index)
    if stream.device_index != index:
        raise ValueError(f"stream: on cuda:{stream.device_index}, the tensors on cuda:{index}")
    return stream.cuda_stream


class PageTables:
    """Block tables of up to max_batch requests and the ring of free pages
    (``cllm_page_tables``): int32 tensors table [max_batch][width], held
    [max_batch], ring [n_pages], state [4] = (first free, free, 0, 0).
    With the table alone the object serves ``PagedCache.attention`` only."""

    def __init__(self, table, held=None, ring=None, state=None, page_size: int = 16):
        if not (isinstance(table, torch.Tensor) and table.dim() == 2):
            raise ValueError("table: need a [max_batch][width] tensor")
        i32, dev = torch.int32, table.get_device() if table.is_cuda else None
        s = _Tables(_tensor(table, "table", i32))
        s.max_batch, s.width = table.shape
        s.page_size = page_size
        if held is not None:
            s.held = _tensor(held, "held", i32, (s.max_batch,), dev)
            s.ring = _tensor(ring, "ring", i32, None, dev)
            s.state = _tensor(state, "state", i32, (4,), dev)
            s.n_pages = ring.numel()
        self.table, self.held, self.ring, self.state, self.page_size = table, held, ring, state, page_size
        self._s, self._p, self._dev = s, ctypes.addressof(s), dev
        self._table, self._width, self._batch = s.table, s.width, s.max_batch

    @classmethod
    def empty(cls, n_pages: int, page_size: int, max_batch: int, width: int, device="cuda"):
        """All pages free, in order."""
        z = dict(dtype=torch.int32, device=device)
        return cls(torch.full((max_batch, width), -1, **z), torch.zeros(max_batch, **z), torch.arange(n_pages, **z),
                   torch.tensor([0, n_pages, 0, 0], **z), page_size)


class PageRows:
    """What a plan says about the step's rows (``cllm_page_rows``): row_start
    [max_batch + 1], seq_len [max_batch], granted [max_batch], positions [max_rows]
    int32 and slots [max_rows] int64.  row_start and seq_len alone serve
    ``PagedCache.attention``.  ``batch``: the requests of the last plan."""

    def __init__(self, row_start, seq_len, granted=None, slots=None, positions=None):
        i32 = torch.int32
        s = _Rows(_tensor(row_start, "row_start", i32))
        dev, n = row_start.get_device(), row_start.numel() - 1
        s.seq_len = _tensor(seq_len, "seq_len", i32, (n,), dev)
        if granted is not None:
            s.granted = _tensor(granted, "granted", i32, (n,), dev)
            s.slots = _tensor(slots, "slots", torch.int64, (slots.numel(),), dev)
            s.positions = _tensor(positions, "positions", i32, (slots.numel(),), dev)
            s.max_rows = slots.numel()
        self.row_start, self.seq_len, self.granted, self.slots, self.positions = row_start, seq_len, granted, slots, positions
        self.batch = n
        self._s, self._p, self._dev = s, ctypes.addressof(s), dev
        self._start, self._len, self._max = s.row_start, s.seq_len, n

    @classmethod
    def empty(cls, max_batch: int, max_rows: int, device="cuda"):
        z = dict(dtype=torch.int32, device=device)
        return cls(torch.zeros(max_batch + 1, **z), torch.zeros(max_batch, **z), torch.zeros(max_batch, **z),
                   torch.full((max_rows,), -1, dtype=torch.int64, device=device), torch.zeros(max_rows, **z))


def plan(tables: PageTables, rows: PageRows, ctx, new_rows, out: Optional[PageTables] = None, stream=None):
    """Pages for requests of ctx cached and new_rows new tokens (int32 [B]) and
    the slots of the new rows (``cllm_page_plan``).  Updates ``tables`` in place, or
    leaves them and fills ``out`` (over the same ring)."""
    out = tables if out is None else out
    if tables.held is None or out.held is None or rows.slots is None:
        raise ValueError("plan needs whole tables and rows")
    dev, b = tables._dev, ctx.numel()
    c = _tensor(ctx, "ctx", torch.int32, None, dev)
    n = _tensor(new_rows, "new_rows", torch.int32, ctx.shape, dev)
    if rows._dev != dev or out._dev != dev or rows._max < b:
        raise ValueError("rows or out: on another device, or too small for the batch")
    args = tables._p, out._p, rows._p, b, c, n, _stream(stream, dev)
    if _device() == dev:
        rc = load().cllm_page_plan(*args)
    else:
        with torch.cuda.device(dev):
            rc = load().cllm_page_plan(*args)
    if rc:
        _c._check(rc, "cllm_page_plan")
    rows.batch = b


class PagedCache:
    """K and V pools [layer][page][kv_head][position][head_dim] of one dtype and
    equal strides, the innermost contiguous (a permuted view gives pages that
    hold one position's heads together), and the scratch of their attention."""

    def __init__(self, k, v, n_heads: int):
        lib = load()
        for t, what in ((k, "k"), (v, "v")):
            if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 5 and t.dtype in DTYPES):
                raise ValueError(f"{what}: need a [layer][page][head][position][head_dim] CUDA tensor of "
                                 "float32, bfloat16 or float16")
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.device != v.device or k.stride(4) != 1:
            raise ValueError("k and v: need the same shape, strides, type and device, head_dim contiguous")
        self.k, self.v, self.n_heads = k, v, n_heads
        self.layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.dtype, self.device = k.dtype, k.device
        d = _Desc(k.data_ptr(), v.data_ptr(), DTYPES[k.dtype], self.layers, self.n_pages, self.page_size,
                  self.n_kv_heads, self.head_dim, n_heads, *k.stride()[:4])
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _c._check(lib.cllm_paged_create(ctypes.byref(d), ctypes.byref(h)), "cllm_paged_create")
        self._h, self._lib, self._dev = h, lib, k.get_device()
        self._args = ctypes.create_string_buffer(max(_ROWS_IN.size, _ATTN.size))
        self._argp = ctypes.addressof(self._args)
        self._scale = self.head_dim ** -0.5

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.cllm_paged_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _heads(self, t, what: str, rows: int, heads: int):
        """Rows of heads side by side: (address, row stride)."""
        hd = self.head_dim
        if isinstance(t, torch.Tensor) and t.dtype is self.dtype and t.get_device() == self._dev and t.shape == (rows, heads, hd):
            row, head, one = t.stride()
            if one == 1 and (head == hd or heads == 1):
                return t.data_ptr(), row
        raise ValueError(f"{what}: need [{rows}][{heads}][{hd}] {self.dtype} on {self.device}, heads side by side")

    def append(self, layer: int, k, v, slots, q=None, q_out=None, rope=None, positions=None, stream=None):
        """Write rows k, v [T][kv_heads][hd] into slots (int64 [T] or more; -1: none).
        With rope (float32 [max_pos][hd/2][2]: cos, sin) K is rotated by positions
        (int32 [T] or more), and q [T][n_heads][hd] into q_out (None: in place)."""
        t = k.shape[0]
        kp, ks = self._heads(k, "k", t, self.n_kv_heads)
        vp, vs = self._heads(v, "v", t, self.n_kv_heads)
        sp = _tensor(slots, "slots", torch.int64, None, self._dev)
        if slots.numel() < t:
            raise ValueError("slots: fewer than rows")
        qp = qs = op = os = rp = pp = max_pos = 0
        if rope is not None:
            max_pos = rope.shape[0]
            rp = _tensor(rope, "rope", torch.float32, (max_pos, self.head_dim // 2, 2), self._dev)
            pp = _tensor(positions, "positions", torch.int32, None, self._dev)
            if positions.numel() < t:
                raise ValueError("positions: fewer than rows")
            if q is not None:
                qp, qs = self._heads(q, "q", t, self.n_heads)
                op, os = (qp, qs) if q_out is None else self._heads(q_out, "q_out", t, self.n_heads)
        elif q is not None:
            raise ValueError("q is only rotated: pass rope")
        _ROWS_IN.pack_into(self._args, 0, layer, t, kp, vp, qp, op, ks, vs, qs, os, sp, rp, pp, max_pos)
        rc = self._lib.cllm_paged_append(self._h, self._argp, _stream(stream, self._dev))
        if rc:
            _c._check(rc, "cllm_paged_append")

    def attention(self, layer: int, q, rows: PageRows, tables: PageTables, out=None, lse=None,
                  scale: Optional[float] = None, window: int = 0, block_mask=None, stream=None):
        """Attention of the step's rows q [T][n_heads][hd] (any row and head stride)
        over their requests' pages; returns out (None: allocated on the stream of the call;
        else no part of q).  lse: float32 [T][n_heads] to fill.
        scale: default head_dim ** -0.5.  window: keys nearer than that (0: all).
        block_mask: int32 [T][words], bit j of word w: the row sees new token 32 w + j of
        its request (None: causal), at least one word."""
        dev, dtype = self._dev, self.dtype
        if out is None:
            # (from the memory of the stream that writes it: the current stream's may still be in use there)
            with nullcontext() if stream is None else torch.cuda.stream(stream):
                out = torch.empty(q.shape, dtype=dtype, device=self.device)
        t = q.shape[0]
        shape = (t, self.n_heads, self.head_dim)
        qs, qh, q1 = q.stride() if q.shape == shape else (0, 0, 0)
        os, oh, o1 = out.stride() if out.shape == shape else (0, 0, 0)
        if not (q1 == 1 and o1 == 1 and q.dtype is dtype and out.dtype is dtype and q.get_device() == dev
                and out.get_device() == dev):
            raise ValueError(f"q and out: need [rows][{self.n_heads}][{self.head_dim}] {dtype} on {self.device}")
        if tables.page_size != self.page_size or rows.batch > tables._batch or tables._dev != dev or rows._dev != dev:
            raise ValueError("rows and tables: another page size or device, or more requests than tables")
        lp = 0 if lse is None else _tensor(lse, "lse", torch.float32, (t, self.n_heads), dev)
        mp = words = 0
        if block_mask is not None:
            words = block_mask.shape[1] if isinstance(block_mask, torch.Tensor) and block_mask.dim() == 2 else 0
            if words == 0:  # (its address would be that of no mask)
                raise ValueError("block_mask: need [rows][words], one word at least")
            mp = _tensor(block_mask, "block_mask", torch.int32, (t, words), dev)
        _ATTN.pack_into(self._args, 0, layer, rows.batch, t, q.data_ptr(), out.data_ptr(), lp, qs, qh, os, oh, rows._start,
                        rows._len, tables._table, tables._width, self._scale if scale is None else scale, window, mp, words)
        rc = self._lib.cllm_paged_attention(self._h, self._argp, _stream(stream, dev))
        if rc:
            _c._check(rc, "cllm_paged_attention")
        return out

    def check(self, stream=None):
        """Wait for the stream; raise CllmError if a call found a page, slot or
        position outside its pool or table, or a wait ran out (and forget it)."""
        _c._check(self._lib.cllm_paged_status(self._h, _stream(stream, self._dev)), "cllm_paged_status")
