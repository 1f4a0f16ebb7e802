"""The 8-bit key/value cache and its attention in plain numpy, 64 bits -- TEST INFRASTRUCTURE ONLY.

Definitions (include/kmq.h, "Key/value cache in 8 bits"); no code shared with the library.  A cache is held as the values
its codes stand for and one multiplier per page and head (the code of x is the one nearest to x * mul).
"""
from __future__ import annotations

import numpy as np

QMAX = {"int8": 127.0, "fp8": 448.0}


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes of e4m3 (4 exponent bits, bias 7, 3 mantissa bits; 0x7f and 0xff are NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if c & 127 == 127:
            x = np.nan
        out[c] = -x if c & 128 else x
    return out


_E4M3 = e4m3_values()[:127]  # 0 .. 448 in rising order: index = code, so even indices are even significands


def nearest_code(y: np.ndarray, fmt: str) -> np.ndarray:
    """The code value nearest to y (|y| at most half a step past the largest), ties to the even code."""
    y = np.asarray(y, dtype=np.float64)
    if fmt == "int8":
        return np.rint(y)
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_E4M3, a), 1, 126)
    lo = hi - 1
    below, above = a - _E4M3[lo], _E4M3[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return np.copysign(np.where(up, _E4M3[hi], _E4M3[lo]), y)


def short(x) -> np.float32:
    """fp32 x without what lies below its eight leading bits (x > 0)."""
    return (np.asarray(x, np.float32).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)


def multiplier(top, fmt: str):
    with np.errstate(divide="ignore", over="ignore"):
        return short(np.minimum(np.float32(QMAX[fmt]) / np.asarray(top, np.float32), np.float32(2.0 ** 100)))


class Cache:
    def __init__(self, fmt, k_codes, v_codes, mul_k, mul_v):
        """k_codes [pages][heads][page][d], v_codes [pages][heads][d][page] (code values); mul float32 [pages][heads]."""
        self.fmt = fmt
        self.codes = [np.array(k_codes, np.float64), np.array(np.swapaxes(v_codes, 2, 3), np.float64)]
        self.mul = [np.array(mul_k, np.float32), np.array(mul_v, np.float32)]
        self.pages, self.heads, self.page, self.d = self.codes[0].shape

    def scales(self, which):
        return np.float32(1.0) / self.mul[which]

    def _seqs(self, table, lens, starts):
        cap = table.shape[1] * self.page
        for b in range(len(lens)):
            n, ln = starts[b + 1] - starts[b], int(lens[b])
            if 0 <= ln <= cap:
                yield b, ln, int(starts[b]), int(n)

    def write(self, table, lens, starts, k, v):
        for b, ln, r0, n in self._seqs(table, lens, starts):
            for p in range(max(0, ln - n) // self.page, -(-ln // self.page)):
                pg = table[b, p]
                i0, i1 = max(ln - n, 0, p * self.page), min(ln, (p + 1) * self.page)
                if i0 >= i1 or not 0 <= pg < self.pages:
                    continue
                for which, x in ((0, k), (1, v)):
                    for h in range(self.heads):
                        part = np.array(x[r0 + i0 - (ln - n):r0 + i1 - (ln - n), h], np.float64)
                        fin = np.where(np.isfinite(part), part, 0.0)
                        top = np.abs(fin).max()
                        part = np.clip(np.where(np.isnan(part), 0.0, part), -top, top)
                        mul = multiplier(top, self.fmt)
                        at = i0 - p * self.page
                        page = self.codes[which][pg, h]
                        if at:
                            was = self.mul[which][pg, h]
                            mul = min(mul, was)
                            if mul < was:
                                page[:at] = nearest_code(page[:at] * float(mul) / float(was), self.fmt)
                        page[at:i1 - p * self.page] = nearest_code(part * float(mul), self.fmt)
                        self.mul[which][pg, h] = mul

    def rows(self, table_row, lo, hi):
        """(keys, values) of positions [lo, hi) as code times scale in fp32 terms, fp64: [n][heads][d]; NaN: no page."""
        out = []
        for which in (0, 1):
            sc = self.scales(which).astype(np.float64)
            x = np.full((hi - lo, self.heads, self.d), np.nan)
            for j in range(lo, hi):
                pg = table_row[j // self.page]
                if 0 <= pg < self.pages:
                    x[j - lo] = self.codes[which][pg, :, j % self.page] * sc[pg][:, None]
            out.append(x)
        return out

    def attend(self, table, lens, starts, q, scale, causal=True, window=0):
        """(out, lse, weighted sum of |v|, largest scale * sum |q||k| a row sees, largest p_j times the largest value of
        page j), fp64; rows of no sequence NaN."""
        rows, hq, d = q.shape
        group = hq // self.heads
        q = np.asarray(q, np.float64)
        o = np.full((rows, hq, d), np.nan)
        lse = np.full((rows, hq), np.nan)
        av = np.zeros((rows, hq, d))
        big = np.zeros((rows, hq))
        most = np.zeros((rows, hq))
        sv = self.scales(1).astype(np.float64) * QMAX[self.fmt]
        for b, ln, r0, n in self._seqs(table, lens, starts):
            k, v = self.rows(table[b], 0, ln)
            j = np.arange(ln)
            there = ~np.isnan(k[:, 0, 0])
            reach = sv[np.where(there, table[b][j // self.page], 0)]
            for i in range(n):
                pos = ln - n + i
                see = there.copy()
                if causal:
                    see &= j <= pos
                if window:
                    see &= j > pos - window
                if not see.any():
                    o[r0 + i] = 0.0
                    lse[r0 + i] = -np.inf
                    continue
                for h in range(hq):
                    kk, vv = k[see, h // group], v[see, h // group]
                    z = scale * (kk @ q[r0 + i, h])
                    top = z.max()
                    e = np.exp(z - top)
                    s = e.sum()
                    o[r0 + i, h] = (e / s) @ vv
                    lse[r0 + i, h] = top + np.log(s)
                    av[r0 + i, h] = (e / s) @ np.abs(vv)
                    most[r0 + i, h] = (e / s * reach[see, h // group]).max()
                    big[r0 + i, h] = scale * (np.abs(kk) @ np.abs(q[r0 + i, h])).max()
        return o, lse, av, big, most
