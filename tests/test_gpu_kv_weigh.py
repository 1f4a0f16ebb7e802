"""kv_weigh where its numbers are far from 1, against the 64-bit oracle (oracle/kv_ops.py).

The bound is that of test_gpu_kv_evict.py: with A the largest scale * sum |q||k| of a row that sees a position, N terms and
e = 2^-24 (d A + 4 T + 8), T = 1.45 A + 16 (the exponent in base 2), (2 e + N 2^-24) of the sum and 12 * 2^-24 of sum p |lse|, for fp32 rows
2^-20 A of the sum more (queries in two halves); of the new weight 2^-23.  Powers of two that queries and keys are multiplied by change no
rounding, so they do not enter.
"""
import math

import numpy as np
import pytest

from gpu_util import host, say, torch_cuda
from test_gpu_kv_evict import _setup, _weights

pytestmark = pytest.mark.gpu

FMTS = ["int8", "fp8", "int4"]

# One for each way in which a call is cut up, by the type of the rows: heads, group, d, lens, rows
WAYS = {
    "tokens": (2, 2, 64, [100, 33], [1, 3]),
    "few": (1, 4, 64, [130, 90], [5, 9]),
    "some": (2, 4, 128, [100, 300], [5, 40]),
    "many": (1, 8, 96, [200, 70], [150, 40]),
}


def _check(s, q, type_, scale, label, decay=0.9):
    import oracle.kv_ops as ops
    scale = float(np.float32(scale))
    _, lse = s.km.kv_attend(s.cache, s.seqs, q, scale=scale, lse=True)
    w, wd = _weights(s)
    s.km.kv_weigh(s.cache, s.seqs, q, lse, wd, scale=scale, decay=decay)
    s.torch.cuda.synchronize()
    got, L = host(wd).astype(np.float64), host(lse)
    assert np.isfinite(L).all(), label
    want, big, els = ops.weigh(s.orc, s.table, s.lens, s.starts, q.float().cpu().numpy(), L, w, scale,
                               decay=float(np.float32(decay)))
    n = s.max_rows * q.shape[1] // s.orc.heads
    e = 2.0 ** -24 * (s.orc.d * big + 4 * (1.45 * big + 16) + 8)
    bound = np.abs(want) * (2 * e + n * 2.0 ** -24 + (2.0 ** -20 * big if type_ == "f32" else 0) + 2.0 ** -23) + \
        12 * 2.0 ** -24 * els + 1e-37
    off = np.abs(got - want)
    assert (off <= bound).all(), f"{label}: {np.nanmax(off):.3e}, {int((~(off <= bound)).sum())} of {off.size} past the bound"


def _keys_times(s, power):
    """Key scales times 2^power, in the cache and the oracle."""
    s.cache.k_scale.mul_(2.0 ** power)
    s.orc.mul[0] *= np.float32(2.0 ** -power)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("type_", ["bf16", "f32"])
@pytest.mark.parametrize("way", list(WAYS))
def test_queries_and_keys_far_from_one(fmt, type_, way):
    """Ordinary scores of queries near the largest number (their products with codes leave fp32's range) and of keys near it."""
    heads, group, d, lens, rows = WAYS[way]
    say(f"kv_weigh far from one {fmt} {type_} {way}")
    large = 125 if fmt == "int4" else 124
    for q_power, k_power in ((large, -20), (-100, 25 if fmt == "int4" else 80)):
        s = _setup(fmt, 32, heads, d, lens, rows, seed=900)
        _keys_times(s, k_power)
        q = s.normal((s.rows, heads * group, d), type_, 0.3 if fmt == "fp8" else 0.5) * 2.0 ** q_power
        assert bool(q.isfinite().all())
        scale = 2.0 ** -(q_power + k_power) / math.sqrt(d)
        _check(s, q, type_, scale, f"queries 2^{q_power}")
        q[1::2] *= 2.0 ** -q_power  # beside rows of ordinary size, whose scores are then next to 0 or too small to count
        if q_power > 0:
            _check(s, q, type_, scale, "mixed")


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("type_", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("way", list(WAYS))
def test_queries_of_zero_over_the_largest_keys(fmt, type_, way):
    """Every score is 0, whatever scores are multiplied by: each position gets its share of one."""
    heads, group, d, lens, rows = WAYS[way]
    say(f"kv_weigh zero queries {fmt} {type_} {way}")
    s = _setup(fmt, 32, heads, d, lens, rows, seed=901)
    s.cache.k_scale.fill_(2.0 ** 119)
    s.orc.mul[0][:] = np.float32(2.0 ** -119)
    q = s.torch.zeros((s.rows, heads * group, d), dtype=s.normal((1,), type_).dtype, device="cuda")
    _check(s, q, type_, 4096.0, "zero")


# As above with sequences that have no rows in the call (lengths, rows): one idle, one idle and empty, one idle that is longer than the others,
# one whose length does not fit.
IDLE = {
    "tokens": (2, 2, 64, [100, 40, 0, 333, 33], [1, 0, 0, 0, 3]),
    "few": (1, 4, 64, [130, 40, 0, 333, 90], [5, 0, 0, 0, 9]),
    "some": (2, 4, 128, [100, 40, 0, 700, 300], [5, 0, 0, 0, 40]),
    "many": (1, 8, 96, [200, 40, 0, 900, 70], [150, 0, 0, 0, 40]),
}


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("type_", ["bf16", "f32"])
@pytest.mark.parametrize("way", list(IDLE))
def test_sequences_without_rows_age_too(fmt, type_, way):
    heads, group, d, lens, rows = IDLE[way]
    say(f"kv_weigh idle sequences {fmt} {type_} {way}")
    s = _setup(fmt, 32, heads, d, lens, rows, seed=902, wide=2)
    q = s.normal((s.rows, heads * group, d), type_, 0.3)
    for decay in (0.9, 1.0, 0.0):
        _check(s, q, type_, 1 / math.sqrt(d), f"decay {decay}", decay)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows", [0, 1, 70])
def test_what_idle_sequences_leave_alone(fmt, rows):
    """Only their own positions change, by one rounding: not those behind the end, on pages that are not there or of lengths that do not
    fit; NaN stays with decay 0.5 and goes with 0.  rows = 0: the whole call has none, and the same holds."""
    torch = torch_cuda()
    s = _setup(fmt, 16, 2, 64, [100, 50, 77, 40], [rows, 0, 0, 0], seed=903, wide=1)
    table, lens = s.table.copy(), [100, 50, 77, 10 ** 6]
    table[2, 1:3] = (-1, 10 ** 6)
    seqs = s.seqs_of(lens, s.starts, table)
    q = s.normal((rows, 8, 64), "bf16")
    lse = torch.zeros((rows, 8), device="cuda")
    w, wd = _weights(s)
    w[s.table[1, 0], 1, 3] = np.nan
    mine = np.zeros(w.shape, bool)
    for b in ((1, 2) if rows else (0, 1, 2)):
        for j in range(lens[b]):
            if 0 <= table[b, j // 16] < s.cache.pages:
                mine[table[b, j // 16], :, j % 16] = True
    first = np.zeros(w.shape, bool)
    first[s.table[0, :7]] = rows > 0  # of the sequence that has rows
    for decay in (0.5, 0.9, 1.0, 0.0):
        wd.copy_(torch.from_numpy(w))
        s.km.kv_weigh(s.cache, seqs, q, lse, wd, decay=decay)
        torch.cuda.synchronize()
        want = np.where(mine, w * np.float32(decay) if decay else np.float32(0), w)
        np.testing.assert_array_equal(np.where(first, 0, host(wd)), np.where(first, 0, want), err_msg=f"decay {decay}")


def test_a_call_without_rows_in_a_graph():
    """Captured, replayed with other lengths; one sequence and many, without starts."""
    torch = torch_cuda()
    s = _setup("int4", 16, 2, 64, [100, 50], [1, 1], seed=904)
    w, wd = _weights(s)
    seqs = s.km.KvSeqs(s.seqs.table, s.seqs.lens, rows=0, max_rows=0)
    q, lse = torch.empty((0, 4, 64), device="cuda"), torch.empty((0, 4), device="cuda")
    s.km.kv_weigh(s.cache, seqs, q, lse, wd, decay=0.5)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.km.kv_weigh(s.cache, seqs, q, lse, wd, decay=0.5)
    for n in (100, 30, 0):
        wd.copy_(torch.from_numpy(w))
        s.seqs.lens.copy_(torch.tensor([n, 50], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want = w.copy()
        for b, ln in enumerate((n, 50)):
            for j in range(ln):
                want[s.table[b, j // 16], :, j % 16] *= np.float32(0.5)
        np.testing.assert_array_equal(host(wd), want)
