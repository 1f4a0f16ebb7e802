"""The key/value cache in 8 bits and the attention over it (kv_write, kv_read, kv_attend of include/kmq.h).

A KvCache is four tensors that the caller owns; a KvSeqs says which rows of a call belong to which sequence.  Both keep the
descriptors that the C ABI takes, so a program that serves makes them once (a KvSeqs once per step, for all layers) and a
call costs little more than its launch.

The cache serves and nothing is trained through it: rows that require grad are refused unless gradients are off.
"""
from __future__ import annotations

import ctypes as ct
import math

import torch

from ._kmq import KmKvCache, KmKvRows, KmKvSeqs, KmqError, _check, _dev, lib

KM_KV_I8, KM_KV_F8 = 0, 1
KM_KV_CAUSAL = 1
_FORMATS = {torch.int8: KM_KV_I8, torch.float8_e4m3fn: KM_KV_F8}
_raw_stream = torch._C._cuda_getCurrentRawStream  # the handle alone: current_stream() makes an object of it first
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _i32(x: int) -> int:
    """A number as the C ABI takes it: one past 32 bits is the largest or -1, not its low half."""
    return max(-1, min(x, 2 ** 31 - 1))


def _beside(t: torch.Tensor, name: str, other: torch.Tensor):
    if t.device != other.device:
        raise ValueError(f"{name} must be on {other.device} (got {t.device})")


class KvCache:
    """Codes and scales of a paged cache (mirrors ``km_kv_cache``).

    k: [pages, heads, page, d] and v: [pages, heads, d, page], int8 or float8_e4m3fn; k_scale, v_scale: float32
    [pages, heads].  value = code * scale.  page is 16, 32, 64 or 128 tokens, d a multiple of 16 up to 256."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if k.dtype not in _FORMATS:
            raise TypeError(f"k must be int8 or float8_e4m3fn (got {k.dtype})")
        _dev(k, k.dtype, "k", 4)
        _dev(v, k.dtype, "v", 4)
        _beside(v, "v", k)
        pages, heads, page, d = k.shape
        if tuple(v.shape) != (pages, heads, d, page):
            raise ValueError("v must be [pages, heads, d, page] for k [pages, heads, page, d]")
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _dev(t, torch.float32, name, 2)
            _beside(t, name, k)
            if tuple(t.shape) != (pages, heads):
                raise ValueError(f"{name} must be [pages, heads]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page, self.d = pages, heads, page, d
        self.device = k.device
        self._c = KmKvCache(_FORMATS[k.dtype], page, heads, d, pages, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                            v_scale.data_ptr())
        self._ref = ct.addressof(self._c)


def kv_cache(pages: int, heads: int, d: int, page: int = 64, dtype: torch.dtype = torch.int8, device="cuda") -> KvCache:
    """A new cache without contents."""
    if dtype not in _FORMATS:
        raise TypeError(f"dtype must be int8 or float8_e4m3fn (got {dtype})")
    k = torch.zeros((pages, heads, page, d), dtype=torch.int8, device=device).view(dtype)
    v = torch.zeros((pages, heads, d, page), dtype=torch.int8, device=device).view(dtype)
    return KvCache(k, v, torch.ones((pages, heads), dtype=torch.float32, device=device),
                   torch.ones((pages, heads), dtype=torch.float32, device=device))


class KvSeqs:
    """The sequences of a call (mirrors ``km_kv_seqs``).

    table: int32 [n, max_pages], the pages of each sequence (one row expanded to n: all of them have the same pages, which
    may be read and attended, not written); lens: int32 [n], tokens of each one, the call's own
    included; starts: int32 [n + 1], rows starts[b] .. starts[b + 1] of a call are the last positions of sequence b, or
    None: rows / n rows each.  rows: rows of all sequences (default n, one each); max_rows: the most of one sequence, of which a
    sequence may not have more (default rows / n without starts; with starts all rows, which suits one prompt and makes 64 single
    tokens almost three times as slow, 552 instead of 205 us for lengths up to 16384: give it); max_len: the longest of lens
    where the program knows it (it chooses launch shapes and no results).  The tensors are read on the device when a call runs and
    may be changed between calls."""

    def __init__(self, table: torch.Tensor, lens: torch.Tensor, starts: torch.Tensor | None = None,
                 rows: int | None = None, max_rows: int | None = None, max_len: int = 0):
        if not isinstance(table, torch.Tensor) or table.device.type != "cuda" or table.dtype != torch.int32 or \
                table.dim() != 2 or table.shape[1] < 1 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table must be a 2-D int32 tensor on the GPU with contiguous rows")
        _dev(lens, torch.int32, "lens", 1)
        _beside(lens, "lens", table)
        n = table.shape[0]
        if lens.shape[0] != n:
            raise ValueError("lens must hold one length per row of table")
        if rows is None:
            rows = n
        if starts is not None:
            _dev(starts, torch.int32, "starts", 1)
            _beside(starts, "starts", table)
            if starts.shape[0] != n + 1:
                raise ValueError("starts must hold n + 1 values")
            max_rows = rows if max_rows is None else max_rows
        else:
            if max_rows is None:
                max_rows = rows // n if n else 0
            if rows != n * max_rows:
                raise ValueError("without starts rows must be n * max_rows")
        ld = table.stride(0)
        if n <= 1:  # the stride of an axis of one is of no meaning
            ld = table.shape[1]
        elif ld != 0 and ld < table.shape[1]:
            raise ValueError(f"table's rows must not overlap in part (stride {ld}, {table.shape[1]} pages)")
        self.table, self.lens, self.starts = table, lens, starts
        self.n, self.rows, self.max_rows, self.max_len = n, rows, max_rows, max_len
        self.device = table.device
        self._c = KmKvSeqs(n, table.shape[1], table.data_ptr(), ld, lens.data_ptr(),
                           None if starts is None else starts.data_ptr(), rows, _i32(max_rows), _i32(max_len))
        self._ref = ct.addressof(self._c)


def _rows_of(t: torch.Tensor, name: str, seqs: KvSeqs, heads: int, d: int, dtype=None, written: bool = False):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in _TYPES or (dtype is not None and t.dtype != dtype):
        raise TypeError(f"{name} must be {dtype or 'float32, bfloat16 or float16'} (got {t.dtype})")
    if t.device != seqs.device:
        raise ValueError(f"{name} must be on {seqs.device} (got {t.device})")
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires grad, and nothing is passed back through the cache: call under torch.no_grad() or "
                         "detach it")
    if t.shape != (seqs.rows, heads, d):
        raise ValueError(f"{name} must be [{seqs.rows}, {heads}, {d}] (got {tuple(t.shape)})")
    row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    if seqs.rows <= 1:  # the stride of an axis of one is of no meaning
        row = 0
    if heads == 1:
        head = 0
    if written and ((row < d and seqs.rows > 1) or (head < d and heads > 1) or
                    (seqs.rows > 1 and heads > 1 and  # the axis of the larger stride steps over the other one
                     (row < (heads - 1) * head + d if row >= head else head < (seqs.rows - 1) * row + d))):
        raise ValueError(f"{name} is written: its rows and heads must not overlap")
    return KmKvRows(t.data_ptr(), row, head)


def _same(cache: KvCache, seqs: KvSeqs):
    if cache.device != seqs.device:
        raise ValueError(f"cache on {cache.device}, sequences on {seqs.device}")


def kv_write(cache: KvCache, seqs: KvSeqs, k: torch.Tensor, v: torch.Tensor) -> None:
    """Puts the rows' keys and values ([rows, heads, d], float32, bfloat16 or float16) into the cache.  A page's scale
    grows with its largest magnitude; the codes of its earlier tokens are then coded again.  NaN counts as 0, an infinity as
    the largest finite magnitude written to its page by the call."""
    _same(cache, seqs)
    kr = _rows_of(k, "k", seqs, cache.heads, cache.d)
    vr = _rows_of(v, "v", seqs, cache.heads, cache.d, k.dtype)
    if seqs.rows:
        _check(lib().kv_write(cache._ref, seqs._ref, ct.addressof(kr), ct.addressof(vr), _TYPES[k.dtype],
                              _raw_stream(cache.device.index)))


def kv_read(cache: KvCache, seqs: KvSeqs, dtype: torch.dtype = torch.bfloat16, k: torch.Tensor | None = None,
            v: torch.Tensor | None = None):
    """The rows' keys and values ([rows, heads, d]) as the cache holds them, rounded to dtype, into k and v where given."""
    _same(cache, seqs)
    if k is None:
        k = cache.k_scale.new_empty((seqs.rows, cache.heads, cache.d), dtype=dtype)
    if v is None:
        v = torch.empty_like(k)
    kr = _rows_of(k, "k", seqs, cache.heads, cache.d, written=True)
    vr = _rows_of(v, "v", seqs, cache.heads, cache.d, k.dtype, written=True)
    if seqs.rows:
        _check(lib().kv_read(cache._ref, seqs._ref, ct.addressof(kr), ct.addressof(vr), _TYPES[k.dtype],
                             _raw_stream(cache.device.index)))
    return k, v


def kv_attend(cache: KvCache, seqs: KvSeqs, q: torch.Tensor, scale: float | None = None, causal: bool = True,
              window: int = 0, out: torch.Tensor | None = None, lse: bool = False):
    """Attention of q ([rows, q_heads, d], q_heads a multiple of the cache's heads) over the cache: (out, lse or None).

    A row sees the positions up to its own (causal) or the whole sequence, with window > 0 the last `window` of them.
    scale: of the products, 1 / sqrt(d) by default.  lse: also the log of each row's sum of exp, float32 [rows, q_heads].
    A row that sees nothing gets zeros and -infinity."""
    _same(cache, seqs)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [rows, q_heads, d]")
    q_heads = q.shape[1]
    qr = _rows_of(q, "q", seqs, q_heads, cache.d)
    if out is None:
        out = torch.empty_like(q)
    orow = _rows_of(out, "out", seqs, q_heads, cache.d, q.dtype, written=True)
    L = q.new_empty((seqs.rows, q_heads), dtype=torch.float32) if lse else None
    if seqs.rows == 0:
        return out, L
    flags = KM_KV_CAUSAL if causal else 0
    t = _TYPES[q.dtype]
    window = _i32(window)
    lb = lib()
    need = lb.kv_attend_bytes(cache._ref, seqs._ref, q_heads, flags, window, t)
    if need < 0:
        raise KmqError(need, lb.km_last_error().decode(errors="replace"))
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _check(lb.kv_attend(cache._ref, seqs._ref, ct.addressof(qr), q_heads,
                        1.0 / math.sqrt(cache.d) if scale is None else scale, flags, window, ct.addressof(orow), t,
                        None if L is None else L.data_ptr(), None if ws is None else ws.data_ptr(), need,
                        _raw_stream(cache.device.index)))
    return out, L
