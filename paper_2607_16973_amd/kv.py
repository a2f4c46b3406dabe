"""Binding of the reader's calls (include/tq.h, "a language model's reader"):
shapes, types and devices are checked here, everything else runs in the
library.  Nothing in this file waits for the GPU except KVCache.check()."""
from __future__ import annotations

import ctypes
import math

import torch

from . import _shape, _stream
from ._lib import (KV_BAD_PAGE, KV_BLOCK, KV_FULL, KV_NONFINITE, KV_PAGE, KV_TYPES, KVCacheView,
                   KVRowsView, RowsView, check, lib)

_CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}
_FLOATS = {torch.float16: 0, torch.bfloat16: 1}
_I32, _F32 = torch.int32, torch.float32


def _on(t, dtype, name, device, ndim):
    """The address of a contiguous tensor of this type on this device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) torch tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != ndim:
        raise ValueError("%s must have %d dimensions" % (name, ndim))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    return t.data_ptr()


def _device(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) torch tensor" % name)
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s is on %s, which is not the current device" % (name, t.device))
    return t.device


def _packed(t, heads, d, name, device, dtype):
    """tq_rows of packed vectors [n, heads, d]; strides are free except the last."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) torch tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    if t.stride(2) != 1 and d > 1:
        raise ValueError("%s: the last dimension must be contiguous" % name)
    return RowsView(t.data_ptr(), t.stride(0), t.stride(1))


def _rank3(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a CUDA (HIP) torch tensor" % name)
    if t.dim() != 3:
        raise ValueError("%s must have shape [tokens, heads, head_dim], got %s" % (name, tuple(t.shape)))


def _float_type(t, name):
    try:
        return _FLOATS[t.dtype]
    except KeyError:
        raise TypeError("%s must be float16 or bfloat16, got %s" % (name, t.dtype)) from None


def _results(q, out, return_lse):
    """out and lse tensors of a call with queries q."""
    n, heads, d = q.shape
    if out is None:
        out = torch.empty((n, heads, d), dtype=q.dtype, device=q.device)
    else:
        _shape(out, (n, heads, d), "out")
        _on(out, q.dtype, "out", q.device, 3)
    lse = torch.empty((n, heads), dtype=_F32, device=q.device) if return_lse else None
    return out, lse


def attention(q, k, v, starts, key_starts=None, *, causal=True, scale=None, longest=0, out=None,
              return_lse=False):
    """Attention over whole prompts of different lengths, packed (tq_attention).

    q [n, heads, d], k and v [n_keys, kv_heads, d]: cuda float16 or bfloat16,
    any strides with a contiguous last dimension; heads a multiple of
    kv_heads; d 64, 128 or 256.  starts (cuda int32 [rows + 1], 0 first)
    bounds each row's queries, key_starts its keys (None: the same).  causal:
    the last query sees every key of its row, each one before it one key
    less; a query that sees none gives 0.  scale: 1/sqrt(d) by default.
    longest: the most queries of a row where the caller knows it.
    Returns out [n, heads, d], with return_lse also the float32 [n, heads]
    logarithm of each query's sum (-inf where it sees no key)."""
    _rank3(q, "q")
    _rank3(k, "k")
    n, heads, d = q.shape
    n_keys, kv_heads = k.shape[0], k.shape[1]
    _shape(k, (n_keys, kv_heads, d), "k")
    _shape(v, (n_keys, kv_heads, d), "v")
    dev, dt = _device(q, "q"), _float_type(q, "q")
    qv = _packed(q, heads, d, "q", dev, q.dtype)
    kv = _packed(k, kv_heads, d, "k", dev, q.dtype)
    vv = _packed(v, kv_heads, d, "v", dev, q.dtype)
    at = _on(starts, _I32, "starts", dev, 1)
    rows = starts.shape[0] - 1
    if rows < 0:
        raise ValueError("starts must have rows + 1 entries")
    kat = None
    if key_starts is not None:
        _shape(key_starts, (rows + 1,), "key_starts")
        kat = _on(key_starts, _I32, "key_starts", dev, 1)
    out, lse = _results(q, out, return_lse)
    check(lib.tq_attention(ctypes.byref(qv), ctypes.byref(kv), ctypes.byref(vv), dt, n, n_keys,
                           heads, kv_heads, d, at, kat, rows, longest, int(causal),
                           1.0 / math.sqrt(d) if scale is None else scale, out.data_ptr(),
                           lse.data_ptr() if return_lse else None, _stream(dev)))
    return (out, lse) if return_lse else out


class KVCache:
    """Keys and values in 8-bit codes with a float32 scale per 16 tokens and
    head, in pages of 64 tokens (tq_kv_cache):

        k        [layers, pages, kv_heads, 64, d]      int8 or float8_e4m3fn
        v        [layers, pages, kv_heads, 4, d, 16]
        k_scale  [layers, pages, kv_heads, 4]          float32; v_scale too
        status   [1] int32: conditions that the kernels met (see check())

    Which pages belong to which row is the caller's (KVPages)."""

    def __init__(self, layers: int, pages: int, kv_heads: int, head_dim: int, dtype: str = "int8",
                 device="cuda"):
        if dtype not in _CODES:
            raise ValueError("dtype must be 'int8' or 'fp8', got %r" % (dtype,))
        # codes and scales of blocks that hold no token are never used, so
        # only the status needs a value
        tiles = (layers, pages, kv_heads)
        k = torch.empty(tiles + (KV_PAGE, head_dim), dtype=_CODES[dtype], device=device)
        v = torch.empty(tiles + (KV_PAGE // KV_BLOCK, head_dim, KV_BLOCK), dtype=_CODES[dtype], device=device)
        scales = [torch.empty(tiles + (KV_PAGE // KV_BLOCK,), dtype=_F32, device=device) for _ in range(2)]
        self._adopt(k, v, scales[0], scales[1], torch.zeros(1, dtype=_I32, device=device))

    @classmethod
    def over(cls, k, v, k_scale, v_scale, status=None) -> "KVCache":
        """A cache over tensors that the caller has (shapes as above)."""
        self = cls.__new__(cls)
        self._adopt(k, v, k_scale, v_scale, status)
        return self

    def _adopt(self, k, v, k_scale, v_scale, status) -> None:
        if not isinstance(k, torch.Tensor) or k.dim() != 5:
            raise ValueError("k must be a tensor [layers, pages, kv_heads, 64, d]")
        layers, pages, heads, page, d = k.shape
        _shape(k, (layers, pages, heads, KV_PAGE, d), "k")
        _shape(v, (layers, pages, heads, KV_PAGE // KV_BLOCK, d, KV_BLOCK), "v")
        _shape(k_scale, (layers, pages, heads, KV_PAGE // KV_BLOCK), "k_scale")
        _shape(v_scale, (layers, pages, heads, KV_PAGE // KV_BLOCK), "v_scale")
        _shape(status, (1,), "status")
        for name, dt in _CODES.items():
            if k.dtype == dt:
                self.dtype = name
                break
        else:
            raise TypeError("k must be int8 or float8_e4m3fn, got %s" % k.dtype)
        dev = _device(k, "k")
        self.k, self.v, self.k_scale, self.v_scale, self.status = k, v, k_scale, v_scale, status
        self.layers, self.pages, self.kv_heads, self.head_dim, self.device = layers, pages, heads, d, dev
        self._view = KVCacheView(_on(k, k.dtype, "k", dev, 5), _on(v, k.dtype, "v", dev, 6),
                                 _on(k_scale, _F32, "k_scale", dev, 4),
                                 _on(v_scale, _F32, "v_scale", dev, 4),
                                 None if status is None else _on(status, _I32, "status", dev, 1),
                                 pages, layers, heads, d, KV_TYPES[self.dtype])
        self._ref = ctypes.byref(self._view)

    def check(self) -> None:
        """Waits for the GPU and raises RuntimeError for the conditions that
        the kernels met since the last check (they are cleared)."""
        if self.status is None:
            raise ValueError("the cache has no status tensor")
        bits = int(self.status.item())
        self.status.zero_()
        said = [text for bit, text in ((KV_NONFINITE, "an appended value was infinite or NaN"),
                                       (KV_BAD_PAGE, "a page id outside the pool was named"),
                                       (KV_FULL, "a row did not get the pages it asked for"))
                if bits & bit]
        if said:
            raise RuntimeError("; ".join(said))

    def _rows(self, tables, lens, starts, n):
        rows = lens.shape[0]
        if not isinstance(tables, torch.Tensor) or tables.dim() != 2:
            raise ValueError("tables must be a tensor [rows, width]")
        _shape(tables, (rows, tables.shape[1]), "tables")
        if starts is None:
            if n != rows:
                raise ValueError("without starts there is one token per row: %d tokens, %d rows" % (n, rows))
        else:
            _shape(starts, (rows + 1,), "starts")
        return (_on(tables, _I32, "tables", self.device, 2), tables.shape[1],
                _on(lens, _I32, "lens", self.device, 1),
                None if starts is None else _on(starts, _I32, "starts", self.device, 1), rows)

    def append(self, layer: int, k, v, tables, lens, starts=None) -> None:
        """Quantises new tokens into one layer (tq_kv_append).  k, v: cuda
        float16 or bfloat16 [n, kv_heads, d], packed by rows, any strides with a contiguous
        last dimension.  tables int32 [rows, width], lens int32 [rows] (the
        new tokens included), starts int32 [rows + 1] (None: one per row)."""
        _rank3(k, "k")
        n = k.shape[0]
        _shape(k, (n, self.kv_heads, self.head_dim), "k")
        _shape(v, (n, self.kv_heads, self.head_dim), "v")
        dt = _float_type(k, "k")
        kv = _packed(k, self.kv_heads, self.head_dim, "k", self.device, k.dtype)
        vv = _packed(v, self.kv_heads, self.head_dim, "v", self.device, k.dtype)
        table, width, length, at, rows = self._rows(tables, lens, starts, n)
        check(lib.tq_kv_append(self._ref, layer, ctypes.byref(kv), ctypes.byref(vv), dt, n, table, width,
                               length, at, rows, _stream(self.device)))

    def attend(self, layer: int, q, tables, lens, starts=None, *, scale=None, longest=0, out=None,
               return_lse=False, workspace=None):
        """Attention of new tokens over one layer of the cache (tq_kv_attend).

        q: cuda float16 or bfloat16 [n, heads, d], the rows' last tokens (one
        each without starts), heads a multiple of kv_heads; tables, lens and
        starts as in append().  A token sees its row up to itself.  longest:
        a bound on lens where the caller has one (it decides how rows are split among workgroups).
        workspace: a cuda uint8 tensor to use instead of a new one.
        Returns out [n, heads, d], with return_lse also the float32 [n, heads]
        logarithm of each query's sum (-inf, and out 0, for a row of length 0)."""
        _rank3(q, "q")
        n, heads, d = q.shape
        _shape(q, (n, heads, self.head_dim), "q")
        dt = _float_type(q, "q")
        qv = _packed(q, heads, d, "q", self.device, q.dtype)
        table, width, length, at, rows = self._rows(tables, lens, starts, n)
        need = ctypes.c_size_t()
        check(lib.tq_kv_attend_workspace(self._ref, n, heads, width, rows, longest, ctypes.byref(need)))
        if workspace is None:
            if need.value:
                workspace = torch.empty((need.value,), dtype=torch.uint8, device=self.device)
        else:
            _on(workspace, torch.uint8, "workspace", self.device, 1)
        out, lse = _results(q, out, return_lse)
        check(lib.tq_kv_attend(self._ref, layer, ctypes.byref(qv), dt, n, heads, table, width, length, at,
                               rows, longest, 1.0 / math.sqrt(d) if scale is None else scale,
                               out.data_ptr(), lse.data_ptr() if return_lse else None,
                               None if workspace is None else workspace.data_ptr(),
                               0 if workspace is None else workspace.numel(), _stream(self.device)))
        return (out, lse) if return_lse else out


class KVPages:
    """The page tables of a batch's rows and the pool's reference counts, on
    the device (tq_kv_rows): tables int32 [rows, width] (-1: no page), lens
    int32 [rows], refs int32 [pages] (rows that hold a page, 0: free)."""

    def __init__(self, rows: int, width: int, pages: int, device="cuda"):
        self._adopt(torch.full((rows, width), -1, dtype=_I32, device=device),
                    torch.zeros(rows, dtype=_I32, device=device),
                    torch.zeros(pages, dtype=_I32, device=device))

    @classmethod
    def over(cls, tables, lens, refs) -> "KVPages":
        """Bookkeeping over tensors that the caller has."""
        self = cls.__new__(cls)
        self._adopt(tables, lens, refs)
        return self

    def _adopt(self, tables, lens, refs) -> None:
        if not isinstance(tables, torch.Tensor) or tables.dim() != 2:
            raise ValueError("tables must be a tensor [rows, width]")
        rows, width = tables.shape
        _shape(lens, (rows,), "lens")
        dev = _device(tables, "tables")
        self.tables, self.lens, self.refs, self.device = tables, lens, refs, dev
        self._view = KVRowsView(_on(tables, _I32, "tables", dev, 2), _on(lens, _I32, "lens", dev, 1),
                                _on(refs, _I32, "refs", dev, 1), refs.shape[0], rows, width)
        self._ref = ctypes.byref(self._view)

    def _workspace(self, n: int):
        need = ctypes.c_size_t()
        check(lib.tq_kv_rows_workspace(self._ref, n, ctypes.byref(need)))
        return torch.empty((need.value,), dtype=torch.uint8, device=self.device)

    def resize(self, goals, cache: KVCache) -> None:
        """Sets the rows' lengths to goals (int32 [rows], negative: leave):
        shrinking rows give pages back, growing ones take the lowest free
        pages in row order (tq_kv_resize).  A row that does not get its pages
        stays as it is, and cache.check() says so."""
        _shape(goals, tuple(self.lens.shape), "goals")
        at = _on(goals, _I32, "goals", self.device, 1)
        ws = self._workspace(0)
        check(lib.tq_kv_resize(self._ref, at, cache._ref, ws.data_ptr(), ws.numel(), _stream(self.device)))

    def fork(self, src, dst, cache: KVCache) -> None:
        """Makes rows dst (int32 [n], distinct) copies of rows src (int32
        [n]): whole pages are shared, a part-filled one is copied in every
        layer (tq_kv_fork)."""
        if not isinstance(src, torch.Tensor) or src.dim() != 1:
            raise ValueError("src must be a tensor [n]")
        _shape(dst, tuple(src.shape), "dst")
        a, b = _on(src, _I32, "src", self.device, 1), _on(dst, _I32, "dst", self.device, 1)
        ws = self._workspace(src.shape[0])
        check(lib.tq_kv_fork(self._ref, a, b, src.shape[0], cache._ref, ws.data_ptr(), ws.numel(),
                             _stream(self.device)))

    def compact(self, cache: KVCache):
        """Moves the live pages to the front of the pool and returns their
        number (cuda int32 [1]); the pages from there on are free (tq_kv_compact)."""
        live = torch.empty(1, dtype=_I32, device=self.device)
        ws = self._workspace(0)
        check(lib.tq_kv_compact(self._ref, cache._ref, live.data_ptr(), ws.data_ptr(), ws.numel(),
                                _stream(self.device)))
        return live
