"""What goes on around the key/value cache in plain numpy, 64 bits -- TEST INFRASTRUCTURE ONLY.

Definitions (include/kmq.h, "Key/value cache in 8 and 4 bits" and "Around the cache"); no code shared with the library: the cache in
4 bits, rotary positions, the attention weight of cached tokens and eviction by it.
"""
from __future__ import annotations

import numpy as np

from .kv import Cache, nearest_code, short


def multiplier4(top):
    with np.errstate(divide="ignore", over="ignore"):
        m = np.clip(np.float32(7) / np.asarray(top, np.float32), np.float32(2.0 ** -30), np.float32(2.0 ** 30))
        return short(m)


def pack4(x: np.ndarray) -> np.ndarray:
    """Bytes of code values -7 .. 7 along the last axis."""
    u = (np.asarray(x) + 8).astype(np.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def unpack4(b: np.ndarray) -> np.ndarray:
    out = np.empty(b.shape[:-1] + (2 * b.shape[-1],))
    out[..., 0::2] = (b & 15).astype(np.float64) - 8
    out[..., 1::2] = (b >> 4).astype(np.float64) - 8
    return out


class Cache4(Cache):
    """codes [2] of [pages][heads][page][d] (code values), mul [2] of float32 [pages][heads][page]."""

    def __init__(self, k_codes, v_codes, mul_k, mul_v):
        self.fmt = "int4"
        self.codes = [np.array(k_codes, np.float64), np.array(np.swapaxes(v_codes, 2, 3), np.float64)]
        self.mul = [np.array(mul_k, np.float32), np.array(mul_v, np.float32)]
        self.pages, self.heads, self.page, self.d = self.codes[0].shape

    def write(self, table, lens, starts, k, v):
        for b, ln, r0, n in self._seqs(table, lens, starts):
            for i in range(n):
                pos = ln - n + i
                if pos < 0 or not 0 <= table[b, pos // self.page] < self.pages:
                    continue
                pg, tok = table[b, pos // self.page], pos % self.page
                for which, x in ((0, k), (1, v)):
                    row = np.array(x[r0 + i], np.float64)  # heads, d
                    top = np.abs(np.where(np.isfinite(row), row, 0.0)).max(1)
                    row = np.clip(np.where(np.isnan(row), 0.0, row), -top[:, None], top[:, None])
                    mul = multiplier4(top)
                    self.codes[which][pg, :, tok] = np.clip(np.rint(row * mul[:, None].astype(np.float64)), -7, 7)
                    self.mul[which][pg, :, tok] = mul

    def rows(self, table_row, lo, hi):
        out = []
        for which in (0, 1):
            sc = self.scales(which).astype(np.float64)
            x = np.full((hi - lo, self.heads, self.d), np.nan)
            for j in range(lo, hi):
                pg = table_row[j // self.page]
                if 0 <= pg < self.pages:
                    x[j - lo] = self.codes[which][pg, :, j % self.page] * sc[pg, :, j % self.page][:, None]
            out.append(x)
        return out

    def attend(self, table, lens, starts, q, scale, causal=True, window=0):
        """As Cache.attend; the last result is the largest p_j times the largest value that token j can have."""
        rows, hq, d = q.shape
        group = hq // self.heads
        q = np.asarray(q, np.float64)
        o, lse = np.full((rows, hq, d), np.nan), np.full((rows, hq), np.nan)
        av, big, most = np.zeros((rows, hq, d)), np.zeros((rows, hq)), np.zeros((rows, hq))
        sv = 7 * self.scales(1).astype(np.float64)
        for b, ln, r0, n in self._seqs(table, lens, starts):
            if n == 0:
                continue
            k, v = self.rows(table[b], 0, ln)
            j = np.arange(ln)
            there = ~np.isnan(k[:, 0, 0]) if ln else np.zeros(0, bool)
            pos = ln - n + np.arange(n)
            see = np.broadcast_to(there, (n, ln)).copy()
            if causal:
                see &= j <= pos[:, None]
            if window:
                see &= j > pos[:, None] - window
            any_ = see.any(1)
            o[r0:r0 + n][~any_], lse[r0:r0 + n][~any_] = 0.0, -np.inf
            if not any_.any():
                continue
            pg = np.where(there, np.asarray(table)[b][j // self.page], 0)
            for h in range(hq):
                kk, vv = np.nan_to_num(k[:, h // group]), np.nan_to_num(v[:, h // group])
                z = np.where(see, scale * (q[r0:r0 + n, h] @ kk.T), -np.inf)[any_]
                top = z.max(1, keepdims=True)
                e = np.exp(z - top)
                s = e.sum(1, keepdims=True)
                at = r0 + np.nonzero(any_)[0]
                o[at, h], lse[at, h] = (e / s) @ vv, (top + np.log(s))[:, 0]
                av[at, h] = (e / s) @ np.abs(vv)
                most[at, h] = (e / s * sv[pg, h // group, j % self.page]).max(1)
                big[at, h] = scale * np.where(see, np.abs(q[r0:r0 + n, h]) @ np.abs(kk).T, 0.0)[any_].max(1)
        return o, lse, av, big, most


def rotate(x, pos, freq, dims, layout, inverse=False, amplitude=1.0):
    """x [rows][heads][d] turned by positions pos [rows]; the turns are reduced as whole numbers and fractions apart."""
    x = np.array(x, np.float64)
    out = x.copy()
    ang = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)
    z = np.exp(1j * (-ang if inverse else ang))[:, None] * amplitude
    i = np.arange(dims // 2)
    a, b = (i, i + dims // 2) if layout == "halves" else (2 * i, 2 * i + 1)
    w = (x[..., a] + 1j * x[..., b]) * z
    out[..., a], out[..., b] = w.real, w.imag
    return out


def weigh(cache, table, lens, starts, q, lse, weight, scale, causal=True, window=0, decay=1.0):
    """(new weights [pages][heads][page], the largest scale * sum |q||k| of a row that adds to it, sum over rows of p times their
    |lse|): fp64."""
    rows, hq, d = q.shape
    group = hq // cache.heads
    q, lse = np.asarray(q, np.float64), np.asarray(lse, np.float64)
    out = np.array(weight, np.float64)
    big, els = np.zeros_like(out), np.zeros_like(out)
    for b, ln, r0, n in cache._seqs(table, lens, starts):
        if ln == 0:
            continue
        k, _ = cache.rows(table[b], 0, ln)
        j = np.arange(ln)
        there = ~np.isnan(k[:, 0, 0])
        pos = ln - n + np.arange(n)
        see = np.ones((n, ln), bool)
        if causal:
            see &= j <= pos[:, None]
        if window:
            see &= j > pos[:, None] - window
        pg, tok = np.where(there, np.asarray(table)[b][j // cache.page], 0), j % cache.page
        for h in range(cache.heads):
            kk = np.nan_to_num(k[:, h])
            total, wide, far = np.zeros(ln), np.zeros(ln), np.zeros(ln)
            for hh in range(h * group, (h + 1) * group):
                L = lse[r0:r0 + n, hh]
                ok = np.isfinite(L)
                if not ok.any():
                    continue
                qq = np.where(ok[:, None], q[r0:r0 + n, hh], 0.0)
                z = np.where(see & ok[:, None], scale * (qq @ kk.T) - np.where(ok, L, 0.0)[:, None], -np.inf)
                p = np.exp(z)
                total += p.sum(0)
                a = scale * np.abs(qq) @ np.abs(kk).T
                wide = np.maximum(wide, np.where(p > 0, a, 0.0).max(0))
                far += (p * np.abs(np.where(ok, L, 0.0))[:, None]).sum(0)
            t = there
            old = np.where((j >= ln - n) | (decay == 0), 0.0, decay * np.nan_to_num(out[pg, h, tok]) if decay else 0.0)
            out[pg[t], h, tok[t]] = (old + total)[t]
            big[pg[t], h, tok[t]] = wide[t]
            els[pg[t], h, tok[t]] = far[t]
    return out, big, els


def evict(cache, table, lens, weight, keep, max_keep, first=0, recent=0):
    """Moves the kept tokens of every sequence in cache and weight (both changed): (kept [n][heads][max_keep], lens)."""
    n = len(lens)
    kept = np.full((n, cache.heads, max_keep), -1, np.int64)
    left = np.array(lens, np.int64)
    for b in range(n):
        ln = int(lens[b])
        row = np.asarray(table)[b]
        need = -(-ln // cache.page) if ln > 0 else 0
        if not 0 <= ln <= len(row) * cache.page or not all(0 <= p < cache.pages for p in row[:need]):
            continue
        K = min(ln, max(0, min(int(keep[b]), max_keep)))
        left[b] = K
        j = np.arange(ln)
        pg, tok = row[j // cache.page], j % cache.page
        for h in range(cache.heads):
            w = np.asarray(weight, np.float64)[pg, h, tok]
            whole = (j < first) | (j >= ln - recent)
            nan = np.isnan(w)
            # least to most important: NaN, weights, protected; the lower position wins ties
            rank = sorted(range(ln), key=lambda i: (not whole[i], bool(nan[i]), 0.0 if nan[i] or whole[i] else -w[i], i))
            idx = np.array(sorted(rank[:K]), np.int64)
            kept[b, h, :K] = idx
            if K == 0:
                continue
            weight[pg[:K], h, tok[:K]] = weight[pg[idx], h, tok[idx]].copy()
            for which in (0, 1):
                codes = cache.codes[which][pg[idx], h, tok[idx]].copy()
                if cache.fmt == "int4":
                    mul = cache.mul[which][pg[idx], h, tok[idx]].copy()
                    cache.codes[which][pg[:K], h, tok[:K]] = codes
                    cache.mul[which][pg[:K], h, tok[:K]] = mul
                    continue
                was = cache.mul[which][pg[idx], h].astype(np.float64)
                least = np.array([was[t * cache.page:(t + 1) * cache.page].min() for t in range(-(-K // cache.page))])
                new = least[np.arange(K) // cache.page]
                again = new < was
                codes[again] = nearest_code(codes[again] * new[again, None] / was[again, None], cache.fmt)
                cache.codes[which][pg[:K], h, tok[:K]] = codes
                cache.mul[which][row[:len(least)], h] = least.astype(np.float32)
    return kept, left
