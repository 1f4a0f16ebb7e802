"""The key/value cache in 8 and 4 bits and what goes on around it (kv_write, kv_read, kv_attend, kv_rotate, kv_weigh and kv_evict of
include/kmq.h).

A KvCache is four tensors that the caller owns; a KvSeqs says which rows of a call belong to which sequence.  Both keep the
descriptors that the C ABI takes, so a program that serves makes them once (a KvSeqs once per step, for all layers) and a
call costs little more than its launch.

The cache serves and nothing is trained through it: rows that require grad are refused unless gradients are off.
"""
from __future__ import annotations

import ctypes as ct
import math

import torch

from ._kmq import KmKvCache, KmKvRotary, KmKvRows, KmKvSeqs, KmqError, _check, _dev, lib

KM_KV_I8, KM_KV_F8, KM_KV_I4 = 0, 1, 4
KM_KV_CAUSAL = 1
KM_ROT_INVERSE = 1
_FORMATS = {torch.int8: KM_KV_I8, torch.float8_e4m3fn: KM_KV_F8, torch.uint8: KM_KV_I4}
_LAYOUTS = {"halves": 0, "pairs": 1}
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
    [pages, heads].  value = code * scale.  page is 16, 32, 64 or 128 tokens, d a multiple of 16 up to 256.

    4-bit codes (-7 .. 7, held as code + 8, the even dim or token in the low half of its byte): uint8 [pages, heads, page, d / 2]
    and [pages, heads, d, page / 2], a scale for each token, [pages, heads, page]; d a multiple of 32."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if k.dtype not in _FORMATS:
            raise TypeError(f"k must be int8, float8_e4m3fn or uint8 (4-bit codes) (got {k.dtype})")
        _dev(k, k.dtype, "k", 4)
        _dev(v, k.dtype, "v", 4)
        _beside(v, "v", k)
        pages, heads, page, d = k.shape
        if k.dtype == torch.uint8:
            d *= 2
            if tuple(v.shape) != (pages, heads, d, page // 2):
                raise ValueError("v must be [pages, heads, d, page / 2] for k [pages, heads, page, d / 2]")
        elif tuple(v.shape) != (pages, heads, d, page):
            raise ValueError("v must be [pages, heads, d, page] for k [pages, heads, page, d]")
        scales = (pages, heads, page) if k.dtype == torch.uint8 else (pages, heads)
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _dev(t, torch.float32, name, len(scales))
            _beside(t, name, k)
            if tuple(t.shape) != scales:
                raise ValueError(f"{name} must be [pages, heads{', page' if len(scales) == 3 else ''}]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page, self.d = pages, heads, page, d
        self.device = k.device
        self._c = KmKvCache(_FORMATS[k.dtype], page, heads, d, pages, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                            v_scale.data_ptr())
        self._ref = ct.addressof(self._c)


def kv_cache(pages: int, heads: int, d: int, page: int = 64, dtype: torch.dtype = torch.int8, device="cuda") -> KvCache:
    """A new cache without contents (dtype: int8, float8_e4m3fn, or uint8 for 4-bit codes)."""
    if dtype not in _FORMATS:
        raise TypeError(f"dtype must be int8, float8_e4m3fn or uint8 (4-bit codes) (got {dtype})")
    if dtype == torch.uint8:
        if d % 2 or page % 2:
            raise ValueError(f"d = {d} and page = {page} must be even for 4-bit codes")
        k = torch.full((pages, heads, page, d // 2), 0x88, dtype=dtype, device=device)
        v = torch.full((pages, heads, d, page // 2), 0x88, dtype=dtype, device=device)
        return KvCache(k, v, torch.ones((pages, heads, page), dtype=torch.float32, device=device),
                       torch.ones((pages, heads, page), dtype=torch.float32, device=device))
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
    if seqs.rows == 0:  # strides of nothing are of no meaning
        return KmKvRows(t.data_ptr(), 0, 0)
    row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    if seqs.rows == 1:  # the stride of an axis of one is of no meaning
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
    the largest finite magnitude written to its page by the call.  4-bit codes: the same for each token and head by itself, and
    nothing is coded again."""
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


class KvRotary:
    """Rotary positions (mirrors ``km_kv_rotary``).

    freq: float64 [dims / 2] on the GPU, radians per position of each pair of the first dims dims of a head; layout: "halves" (dims i
    and i + dims / 2 are a pair) or "pairs" (2 i and 2 i + 1); amplitude: what sine and cosine are multiplied by.  kv_rotary makes the
    usual frequencies."""

    def __init__(self, freq: torch.Tensor, layout: str = "halves", amplitude: float = 1.0):
        _dev(freq, torch.float64, "freq", 1)
        if layout not in _LAYOUTS:
            raise ValueError(f'layout must be "halves" or "pairs" (got {layout!r})')
        self.freq, self.layout, self.amplitude = freq, layout, float(amplitude)
        self.dims = 2 * freq.shape[0]
        self.device = freq.device
        self._c = KmKvRotary(self.dims, _LAYOUTS[layout], freq.data_ptr(), self.amplitude)
        self._ref = ct.addressof(self._c)


def kv_rotary(dims: int, base: float = 10000.0, layout: str = "halves", scaling: str | None = None, factor: float = 1.0,
              original: int = 0, low: float = 1.0, high: float = 32.0, amplitude: float = 1.0, device="cuda") -> KvRotary:
    """Rotary positions with frequencies base^(-2 i / dims), for longer contexts than they were made for with

    scaling "linear": all of them divided by factor;
    scaling "base": the base times factor^(dims / (dims - 2)), so that the slowest pair is slowed by factor and the fastest not at all;
    scaling "parts": by factor those that turn less than `low` times within `original` positions, not at all those that turn more than
    `high` times, in between in proportion to their number of turns."""
    if dims < 2 or dims % 2:
        raise ValueError(f"dims must be even and at least 2 (got {dims})")
    if not base > 0 or not factor > 0 or not math.isfinite(base) or not math.isfinite(factor):
        raise ValueError(f"base and factor must be finite and > 0 (got {base}, {factor})")
    if scaling not in (None, "linear", "base", "parts"):
        raise ValueError(f'scaling must be None, "linear", "base" or "parts" (got {scaling!r})')
    if scaling == "parts" and (original < 1 or not high > low):
        raise ValueError(f"parts needs original >= 1 and high > low (got {original}, {low}, {high})")
    if scaling == "base":
        if dims == 2:
            raise ValueError("scaling of the base needs more than one pair")
        base *= factor ** (dims / (dims - 2))
    freq = torch.tensor([base ** (-2.0 * i / dims) for i in range(dims // 2)], dtype=torch.float64)
    if scaling == "linear":
        freq /= factor
    elif scaling == "parts":
        keep = ((original * freq / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        freq = freq * keep + freq / factor * (1 - keep)
    return KvRotary(freq.to(device), layout, amplitude)


def _extent(t: torch.Tensor):
    """First byte of rows [rows, heads, d] and one past the last."""
    size = t.element_size()
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
    return t.data_ptr(), t.data_ptr() + (last + 1) * size


def _apart(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether no element of rows a is one of rows b: their ranges are disjoint, or they lie side by side in the same rows."""
    (a0, a1), (b0, b1) = _extent(a), _extent(b)
    if a1 <= b0 or b1 <= a0:
        return True
    step = a.stride(0) * a.element_size()
    if a.shape[0] < 2 or a.stride(0) != b.stride(0):
        return False
    wide = [((t.shape[1] - 1) * t.stride(1) + t.shape[2]) * t.element_size() for t in (a, b)]
    off = (b0 - a0) % step
    return wide[0] <= off and off + wide[1] <= step


def kv_rotate(rotary: KvRotary, at: KvSeqs | torch.Tensor, q: torch.Tensor, k: torch.Tensor | None = None,
              inverse: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """Queries and keys ([rows, heads, d], float32, bfloat16 or float16) turned by their positions: (q, k or None), into q_out and
    k_out where given (q and k themselves: in place).

    at: a KvSeqs, whose rows have the last positions of their sequences, or the positions, int32 [rows].  inverse: turned back, which is
    also how the gradient of a result becomes that of what went in.  A pair (x, y) at position p with frequency f becomes
    (x cos pf - y sin pf, x sin pf + y cos pf)."""
    if isinstance(at, KvSeqs):
        where, seqs, positions = at, at._ref, None
    else:
        _dev(at, torch.int32, "positions", 1)
        where, seqs, positions = _Rows(at.shape[0], at.device), None, at.data_ptr()
    rows = where.rows
    if rotary.device != where.device:
        raise ValueError(f"rotary on {rotary.device}, positions on {where.device}")
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [rows, heads, d]")
    _, q_heads, d = q.shape
    qi = _rows_of(q, "q", where, q_heads, d)
    dtype = q.dtype
    if q_out is None:
        qo_t = q.new_empty((rows, q_heads, d))
        qo = KmKvRows(qo_t.data_ptr(), q_heads * d, d)
    else:
        qo_t, qo = q_out, _rows_of(q_out, "q_out", where, q_heads, d, dtype, written=True)
    ko_t = ki = ko = None
    k_heads = 0
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 3:
            raise ValueError("k must be a tensor [rows, heads, d]")
        k_heads = k.shape[1]
        ki = _rows_of(k, "k", where, k_heads, d, dtype)
        if k_out is None:
            ko_t = k.new_empty((rows, k_heads, d))
            ko = KmKvRows(ko_t.data_ptr(), k_heads * d, d)
        else:
            ko_t, ko = k_out, _rows_of(k_out, "k_out", where, k_heads, d, dtype, written=True)
    elif k_out is not None:
        raise ValueError("k_out without k")
    if rows == 0:
        return qo_t, ko_t
    if q_out is not None or k_out is not None:
        _check_outputs(q, k, q_out, k_out)
    _check(lib().kv_rotate(rotary._ref, seqs, positions, rows, ct.addressof(qi), q_heads, None if k is None else ct.addressof(ki),
                           k_heads, ct.addressof(qo), None if k is None else ct.addressof(ko), d, _TYPES[dtype],
                           KM_ROT_INVERSE if inverse else 0, _raw_stream(where.device.index)))
    return qo_t, ko_t


def _same_rows(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether rows a and b, of one shape, lie in the same places (the stride of an axis of one is of no meaning)."""
    return a.data_ptr() == b.data_ptr() and all(n == 1 or s == z for n, s, z in zip(a.shape, a.stride(), b.stride()))


def _check_outputs(q, k, q_out, k_out):
    """Rows that are written overlap none of the others, but may be the ones that they are made of."""
    for out, name, own, of_own, other, of_other in ((q_out, "q_out", q, "q", k, "k"), (k_out, "k_out", k, "k", q, "q")):
        if out is None:
            continue
        if not _same_rows(out, own) and not _apart(out, own):
            raise ValueError(f"{name} overlaps {of_own} and is not the same rows")
        if other is not None and not _apart(out, other):
            raise ValueError(f"{name} overlaps {of_other}")
    if q_out is not None and k_out is not None and not _apart(q_out, k_out):
        raise ValueError("q_out and k_out overlap")


class _Rows:
    """What _rows_of asks of sequences."""

    def __init__(self, rows, device):
        self.rows, self.device = rows, device


def _weights(weight: torch.Tensor, cache: KvCache):
    _dev(weight, torch.float32, "weight", 3)
    _beside(weight, "weight", cache.k)
    if tuple(weight.shape) != (cache.pages, cache.heads, cache.page):
        raise ValueError(f"weight must be [{cache.pages}, {cache.heads}, {cache.page}] (got {tuple(weight.shape)})")


def kv_weigh(cache: KvCache, seqs: KvSeqs, q: torch.Tensor, lse: torch.Tensor, weight: torch.Tensor,
             scale: float | None = None, causal: bool = True, window: int = 0, decay: float = 1.0) -> None:
    """Adds the attention weight that every cached token gets from the rows' queries, summed over rows and the query heads of its cache
    head, to `weight` (float32 [pages, heads, page], in place) times decay.

    q, scale, causal and window are those of the kv_attend call that left lse (its log-sum-exp, float32 [rows, q_heads]).  The call's own
    tokens begin with this sum; with decay = 0 all tokens do.  Rows whose lse is not finite add nothing.  Sequences without rows in the
    call age like the others: their weights are multiplied by decay, with decay = 0 cleared.  No two sequences of a call
    may have a page in common, and none may have one twice."""
    _same(cache, seqs)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [rows, q_heads, d]")
    q_heads = q.shape[1]
    qr = _rows_of(q, "q", seqs, q_heads, cache.d)
    _dev(lse, torch.float32, "lse", 2)
    _beside(lse, "lse", cache.k)
    if tuple(lse.shape) != (seqs.rows, q_heads):
        raise ValueError(f"lse must be [{seqs.rows}, {q_heads}] (got {tuple(lse.shape)})")
    _weights(weight, cache)
    lb = lib()
    flags, window, t = KM_KV_CAUSAL if causal else 0, _i32(window), _TYPES[q.dtype]
    need = lb.kv_weigh_bytes(cache._ref, seqs._ref, q_heads, flags, window, t)
    if need < 0:
        raise KmqError(need, lb.km_last_error().decode(errors="replace"))
    ws = torch.empty(need, dtype=torch.uint8, device=cache.device) if need else None
    _check(lb.kv_weigh(cache._ref, seqs._ref, ct.addressof(qr), q_heads, 1.0 / math.sqrt(cache.d) if scale is None else scale,
                       flags, window, t, lse.data_ptr(), weight.data_ptr(), decay, None if ws is None else ws.data_ptr(), need,
                       _raw_stream(cache.device.index)))


def kv_evict(cache: KvCache, seqs: KvSeqs, weight: torch.Tensor, keep: torch.Tensor, max_keep: int, first: int = 0,
             recent: int = 0):
    """Every sequence keeps keep[b] (int32 [n], at most max_keep) of its tokens, each head its own: the first `first`, the last
    `recent`, then those of the largest weight, ties to the lower position.  A keep[b] below first + recent is no error, and then it is
    the most recent ones that go: give each sequence at least that much.  They move to the front of the sequence's pages in their
    order, with their codes, scales and weights: (kept, lens).

    kept: int32 [n, heads, max_keep], the position that each kept token had (-1: none); lens: int32 [n], the sequences' new lengths,
    which the program takes over (``seqs.lens.copy_(lens)``); the pages behind them are free.  Only table and lens of seqs are
    looked at.  Tokens that come later have positions that are no longer their places in the cache: rotary positions are then given
    to kv_rotate as such.  No two sequences of a call may have a page in common, and none may have one twice.  The workspace is about
    as large as the codes of the tokens that are kept."""
    _same(cache, seqs)
    _weights(weight, cache)
    _dev(keep, torch.int32, "keep", 1)
    _beside(keep, "keep", cache.k)
    if keep.shape[0] != seqs.n:
        raise ValueError("keep must hold one number per sequence")
    lb = lib()
    max_keep, first, recent = _i32(max_keep), _i32(first), _i32(recent)
    need = lb.kv_evict_bytes(cache._ref, seqs._ref, max_keep)
    if need < 0:
        raise KmqError(need, lb.km_last_error().decode(errors="replace"))
    kept = torch.empty((seqs.n, cache.heads, max_keep), dtype=torch.int32, device=cache.device)
    lens = torch.empty(seqs.n, dtype=torch.int32, device=cache.device)
    ws = torch.empty(need, dtype=torch.uint8, device=cache.device) if need else None
    _check(lb.kv_evict(cache._ref, seqs._ref, weight.data_ptr(), keep.data_ptr(), max_keep, first, recent, kept.data_ptr(),
                       lens.data_ptr(), None if ws is None else ws.data_ptr(), need, _raw_stream(cache.device.index)))
    return kept, lens
