"""The attention weight of cached tokens and eviction by it, against the 64-bit oracle (oracle/kv_ops.py).

Eviction is compared exactly: positions, lengths, codes, scales, weights.  Weights within a bound made of the roundings: of a
position's sum, with A the largest scale * sum |q||k| of a row that sees it, N terms and e = 2^-24 (d A + 4 T + 8), T = 1.45 A + 16
(the exponent in base 2), (2 e + N 2^-24) of the sum and 12 * 2^-24 of sum p |lse|, for fp32 rows 2^-20 A of the sum more (queries in two
halves); of the new weight 2^-23.
"""
import math

import numpy as np
import pytest

from gpu_util import host, say, torch_cuda
from test_gpu_kv import Setup
from test_gpu_kv_int4 import Setup4

pytestmark = pytest.mark.gpu

FMTS = ["int8", "fp8", "int4"]


def _setup(fmt, page, heads, d, lens, rows, seed, **kw):
    return Setup4(page, heads, d, lens, rows, seed, **kw) if fmt == "int4" else Setup(fmt, page, heads, d, lens, rows, seed, **kw)


def _weights(s):
    w = s.rng.gamma(0.3, 2.0, (s.cache.pages, s.cache.heads, s.cache.page)).astype(np.float32)
    return w, s.torch.from_numpy(w).cuda()


def _weigh_check(s, q, type_, causal=True, window=0, decay=1.0, table=None, label=""):
    import oracle.kv_ops as ops
    torch, km = s.torch, s.km
    scale = 1.0 / math.sqrt(s.orc.d)
    seqs = s.seqs if table is None else s.seqs_of(s.lens, s.starts, table)
    _, lse = km.kv_attend(s.cache, seqs, q, causal=causal, window=window, lse=True)
    w, wd = _weights(s)
    km.kv_weigh(s.cache, seqs, q, lse, wd, causal=causal, window=window, decay=decay)
    torch.cuda.synchronize()
    got, L = host(wd).astype(np.float64), host(lse)
    want, big, els = ops.weigh(s.orc, s.table if table is None else table, s.lens, s.starts, q.float().cpu().numpy(), L, w,
                               float(np.float32(scale)), causal, window, float(np.float32(decay)))
    N = s.max_rows * q.shape[1] // s.orc.heads
    e = 2.0 ** -24 * (s.orc.d * big + 4 * (1.45 * big + 16) + 8)
    total = np.abs(want) + 1.0 * 0  # the sum is at most the new weight
    bound = total * (2 * e + N * 2.0 ** -24 + (2.0 ** -20 * big if type_ == "f32" else 0) + 2.0 ** -23) + 12 * 2.0 ** -24 * els + 1e-37
    bad = np.abs(got - want) - bound
    assert bad.max() <= 0, f"{label}: {np.abs(got - want).flat[bad.argmax()]:.3e} bound {bound.flat[bad.argmax()]:.3e}"
    return wd


WEIGHS = [
    # page, heads, group, d, lens, rows, window
    (16, 1, 1, 32, [1], [1], 0),
    (16, 2, 1, 64, [1, 15, 16, 17, 63, 64, 65], [1] * 7, 0),
    (64, 2, 4, 128, [777, 64, 1, 129], [1] * 4, 0),
    (128, 1, 8, 128, [300, 1025], [1, 1], 0),
    (32, 1, 16, 96, [333, 32], [1, 1], 0),
    (64, 2, 2, 192, [129, 500], [1, 1], 0),
    (64, 1, 4, 256, [65, 400], [1, 1], 0),
    (64, 1, 32, 128, [260], [3], 0),
    (32, 2, 3, 160, [50, 40], [7, 40], 0),
    (16, 1, 2, 224, [33, 64], [33, 20], 0),
    (64, 2, 4, 128, [300, 90], [5, 90], 0),
    (64, 1, 4, 64, [200, 130, 3], [130, 130, 3], 0),
    (16, 1, 1, 128, [150], [150], 0),
    (32, 1, 2, 128, [100, 400], [3, 70], 33),
    (64, 2, 8, 128, [1000, 70], [4, 4], 64),
    (64, 1, 1, 64, [500], [1], 1),
    (64, 1, 4, 96, [900, 70], [500, 64], 50),
]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("type_", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", range(len(WEIGHS)))
def test_weigh(fmt, type_, case):
    page, heads, group, d, lens, rows, window = WEIGHS[case]
    say(f"kv_weigh {fmt} {type_} page={page} heads={heads}x{group} d={d} lens={lens} rows={rows} window={window}")
    s = _setup(fmt, page, heads, d, lens, rows, seed=500 + case)
    q = s.normal((s.rows, heads * group, d), type_, 0.3 if fmt == "fp8" else 0.6)
    for decay in (1.0, 0.0, 0.9):
        _weigh_check(s, q, type_, window=window, decay=decay, label=f"decay {decay}")
    if not window:
        _weigh_check(s, q, type_, causal=False, label="whole")


MANY = [
    # page, heads, group, d, lens, rows, window: 512 rows to a cache head and more
    (16, 1, 8, 128, [150, 70], [150, 70], 0),
    (32, 1, 4, 192, [200], [150], 0),
    (128, 1, 4, 256, [160, 129, 0], [160, 129, 1], 33),
    (64, 2, 16, 32, [300, 40], [33, 40], 0),
    (64, 1, 1, 160, [600, 31], [600, 31], 0),
    (16, 2, 5, 96, [700, 130], [130, 130], 64),
]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_weigh_many_rows(fmt, type_, case):
    page, heads, group, d, lens, rows, window = MANY[case]
    say(f"kv_weigh {fmt} {type_} many rows page={page} heads={heads}x{group} d={d} lens={lens} rows={rows} window={window}")
    s = _setup(fmt, page, heads, d, lens, rows, seed=540 + case, wide=2)
    q = s.normal((s.rows, heads * group, d), type_, 0.3 if fmt == "fp8" else 0.6)
    q[1, 0] = math.nan
    _weigh_check(s, q, type_, window=window, decay=0.9, label="causal")
    _weigh_check(s, q, type_, causal=False, window=0, label="whole")
    table = s.table.copy()
    table[0, 1:3] = -1
    _weigh_check(s, q, type_, window=window, table=table, label="absent pages")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows", [1, 70])
def test_weigh_rows_that_see_nothing_and_absent_pages(fmt, rows):
    """Rows before position 0 and rows of NaN add nothing; absent pages have no weight; nobody else's weight changes."""
    s = _setup(fmt, 16, 1, 64, [0, 40, 100, 33], [rows] * 4, seed=9, wide=2)
    q = s.normal((s.rows, 4, 64), "bf16")
    q[rows, 1] = math.nan
    q[2 * rows, 2, 5] = math.inf
    _weigh_check(s, q, "bf16", label="short")
    table = s.table.copy()
    table[1, :] = -1
    table[2, 1:3] = 10 ** 6
    table[3, 0] = -5
    _weigh_check(s, q, "bf16", table=table, label="absent pages")


@pytest.mark.parametrize("fmt", FMTS)
def test_weigh_ignores_what_lies_behind_the_end(fmt):
    """NaN codes, scales and weights behind the end of a sequence change nothing and stay; with decay 0 earlier ones do not count."""
    torch = torch_cuda()
    for rows in (1, 100):
        s = _setup(fmt, 16, 2, 64, [200, 217], [rows, rows], seed=13, wide=3)
        q = s.normal((s.rows, 4, 64), "f16")
        _, lse = s.km.kv_attend(s.cache, s.seqs, q, lse=True)
        used = np.zeros((s.cache.pages, 16), bool)
        for b, ln in enumerate(s.lens):
            for j in range(ln):
                used[s.table[b, j // 16], j % 16] = True
        free = torch.from_numpy(~used).cuda()
        w = torch.zeros((s.cache.pages, 2, 16), device="cuda")
        s.km.kv_weigh(s.cache, s.seqs, q, lse, w)
        if fmt == "int4":
            s.cache.k_scale[free[:, None].expand(s.cache.k_scale.shape)] = math.nan
        else:
            k = s.cache.k.view(torch.uint8)
            k[free[:, None, :, None].expand(k.shape)] = 0x7F
        w2 = torch.full_like(w, math.nan)
        s.km.kv_weigh(s.cache, s.seqs, q, lse, w2, decay=0.0)
        f = free[:, None].expand(w.shape)
        assert torch.equal(w[~f], w2[~f]) and bool(w2[f].isnan().all())


@pytest.mark.parametrize("fmt", FMTS)
def test_weigh_long_and_any_max_len(fmt):
    """Lengths far past the max_len that was given, and a table much wider than the sequences: the same weights."""
    torch = torch_cuda()
    s = _setup(fmt, 64, 2, 64, [5000, 1, 2049], [1, 1, 1], seed=15, wide=900)
    q = s.normal((3, 4, 64), "bf16")
    _weigh_check(s, q, "bf16", label="long")
    _, lse = s.km.kv_attend(s.cache, s.seqs, q, lse=True)
    got = []
    for max_len in (0, 1, 5000, 10 ** 9):
        seqs = s.km.KvSeqs(s.seqs.table, s.seqs.lens, max_len=max_len)
        w = torch.ones((s.cache.pages, 2, 64), device="cuda")
        s.km.kv_weigh(s.cache, seqs, q, lse, w)
        got.append(w)
    assert all(torch.equal(got[0], w) for w in got[1:])


EVICTS = [
    # page, heads, d, lens, keep, max_keep, first, recent
    (16, 1, 32, [1], [1], 1, 0, 0),
    (16, 2, 64, [1, 16, 17, 40, 0, 33], [5, 5, 5, 5, 5, 5], 5, 0, 0),
    (64, 2, 128, [200, 64, 129], [100, 64, 3], 100, 4, 20),
    (32, 3, 96, [300, 100, 31], [64, 33, 31], 64, 0, 8),
    (128, 2, 256, [300, 127], [130, 100], 140, 2, 0),
    (16, 5, 192, [100, 90], [0, -3], 50, 0, 0),
    (64, 1, 64, [500, 70], [1, 500], 600, 1, 0),
    (16, 2, 32, [9000, 100], [4001, 17], 4001, 16, 100),
    (64, 2, 64, [300], [10], 100, 40, 60),
]


def _evict(s, w, wd, keep, max_keep, first, recent, table=None, lens=None, label=""):
    import oracle.kv_ops as ops
    torch = s.torch
    t = s.table if table is None else table
    ln = s.lens if lens is None else np.asarray(lens, np.int32)
    seqs = s.km.KvSeqs(torch.from_numpy(t).cuda(), torch.from_numpy(ln).cuda())
    kept, left = s.km.kv_evict(s.cache, seqs, wd, torch.tensor(keep, dtype=torch.int32, device="cuda"), max_keep, first, recent)
    torch.cuda.synchronize()
    want, want_left = ops.evict(s.orc, t, ln, w, keep, max_keep, first, recent)
    np.testing.assert_array_equal(host(left), want_left, err_msg=label)
    np.testing.assert_array_equal(host(kept), want, err_msg=label)
    np.testing.assert_array_equal(host(wd), w, err_msg=label)
    s.check_cache(label)
    return kept, left


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", range(len(EVICTS)))
def test_evict(fmt, case):
    page, heads, d, lens, keep, max_keep, first, recent = EVICTS[case]
    say(f"kv_evict {fmt} page={page} heads={heads} d={d} lens={lens} keep={keep} of {max_keep} first={first} recent={recent}")
    s = _setup(fmt, page, heads, d, lens, [1] * len(lens), seed=600 + case)
    w, wd = _weights(s)
    _, left = _evict(s, w, wd, keep, max_keep, first, recent, label="first")
    # again, from what is left
    _evict(s, w, wd, [max(k // 2, 0) for k in keep], max_keep, first, recent, lens=host(left), label="second")


@pytest.mark.parametrize("fmt", FMTS)
def test_evict_special_weights(fmt):
    """Ties, zeros of both signs, infinities, NaN, subnormals, negative weights: ties to the lower position, NaN least."""
    s = _setup(fmt, 16, 2, 32, [120, 64, 200, 50], [1] * 4, seed=31)
    w = s.rng.choice(np.array([0.0, -0.0, 1.0, np.nan, np.inf, -np.inf, 1e-42, -2.0, 3e38, 2.0 ** -126], np.float32),
                     (s.cache.pages, 2, 16)).astype(np.float32)
    w[s.table[3, :4]] = 1.0  # all the same
    _evict(s, w, s.torch.from_numpy(w).cuda(), [50, 30, 170, 7], 170, 3, 5, label="special")


@pytest.mark.parametrize("fmt", FMTS)
def test_evict_leaves_alone(fmt):
    """Sequences whose length does not fit or that miss a page; and everything behind the new end."""
    torch = torch_cuda()
    s = _setup(fmt, 16, 2, 32, [40, 100, 100, 33, 64], [1] * 5, seed=33, wide=2)
    w, wd = _weights(s)
    table = s.table.copy()
    table[1, 3], table[2, 6] = -1, 10 ** 6
    lens = [40, 100, 100, -1, 10 ** 6]
    kept, left = _evict(s, w, wd, [10, 10, 10, 10, 10], 20, 0, 0, table=table, lens=lens, label="alone")
    assert host(left).tolist() == [10, 100, 100, -1, 10 ** 6] and (host(kept)[1:] == -1).all()


# Tables that are wide enough for sequences of 50 thousand tokens: chosen from by several workgroups, whatever the lengths are.
WIDE = 51200


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", range(len(EVICTS)))
def test_evict_in_slices(fmt, case):
    page, heads, d, lens, keep, max_keep, first, recent = EVICTS[case]
    say(f"kv_evict {fmt} in slices page={page} heads={heads} d={d} lens={lens} keep={keep} of {max_keep}")
    s = _setup(fmt, page, heads, d, lens, [1] * len(lens), seed=640 + case, wide=WIDE // page)
    w, wd = _weights(s)
    _, left = _evict(s, w, wd, keep, max_keep, first, recent, label="first")
    _evict(s, w, wd, [max(k // 2, 0) for k in keep], max_keep, first, recent, lens=host(left), label="second")


def test_evict_in_slices_special_and_left_alone():
    """Ties, NaN, infinities; lengths that do not fit and pages that are not there beside sequences of several slices."""
    s = Setup4(16, 2, 32, [17001, 40, 100, 33, 64, 16385], [1] * 6, seed=37, wide=WIDE // 16)
    w = s.rng.choice(np.array([0.0, -0.0, 1.0, np.nan, np.inf, -np.inf, 1e-42, -2.0, 3e38, 2.0 ** -126], np.float32),
                     (s.cache.pages, 2, 16)).astype(np.float32)
    w[s.table[5, :1024]] = 1.0  # all the same, but for the last
    table = s.table.copy()
    table[2, 6] = -1
    lens = [17001, 40, 100, -1, 10 ** 6, 16385]
    kept, left = _evict(s, w, s.torch.from_numpy(w).cuda(), [9000, 10, 10, 10, 10, 8200], 9000, 3, 5, table=table, lens=lens,
                        label="slices")
    assert host(left).tolist() == [9000, 10, 100, -1, 10 ** 6, 8200]


def test_evict_in_slices_in_a_graph():
    """Replayed with other weights and lengths, eager calls in between: the same as an eager call each time."""
    torch = torch_cuda()
    s = Setup4(64, 2, 32, [30000, 900], [1, 1], seed=39, wide=WIDE // 64)
    keep = torch.tensor([20000, 300], dtype=torch.int32, device="cuda")
    wd = _weights(s)[1]
    state = (s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale, wd)
    start = [t.clone() for t in state]

    def step():
        return s.km.kv_evict(s.cache, s.seqs, wd, keep, 20000, 4, 64)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step()
    for i in range(3):
        s.seqs.lens.copy_(torch.tensor([30000 - 5001 * i, 900 - i], dtype=torch.int32))
        start[4] = _weights(s)[1]
        out = []
        for run in (lambda: (g.replay(), held)[1], step):
            for t, x in zip(state, start):
                t.copy_(x)
            got = run()
            torch.cuda.synchronize()
            out.append([t.clone() for t in got + state])
        for a, b in zip(*out):
            assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("type_", ["f16", "f32"])
def test_weigh_many_rows_that_see_nothing_and_absent_pages(fmt, type_):
    """As above with rows of the other types, and more of them than one tile."""
    s = _setup(fmt, 32, 2, 96, [0, 40, 200, 33, 70], [70] * 5, seed=10, wide=2)
    q = s.normal((s.rows, 8, 96), type_)
    q[70, 1] = math.nan
    q[140, 2, 5] = math.inf
    _weigh_check(s, q, type_, label="short")
    table = s.table.copy()
    table[1, :] = -1
    table[2, 1:3] = 10 ** 6
    table[3, 0] = -5
    _weigh_check(s, q, type_, table=table, window=50, label="absent pages")


@pytest.mark.parametrize("type_", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 200])
def test_weigh_rows_and_any_max_len(type_, rows):
    """Lengths past the max_len that was given: what is split over workgroups by it is not, and the sums stay right."""
    import oracle.kv_ops as ops
    torch = torch_cuda()
    s = Setup4(64, 1, 64, [1500, rows, 700], [rows] * 3, seed=17)
    q = s.normal((s.rows, 8, 64), type_)
    _, lse = s.km.kv_attend(s.cache, s.seqs, q, lse=True)
    old = np.zeros((s.cache.pages, 1, 64), np.float32)
    want, big, els = ops.weigh(s.orc, s.table, s.lens, s.starts, q.float().cpu().numpy(), host(lse), old,
                               float(np.float32(1 / math.sqrt(64))))
    e = 2.0 ** -24 * (64 * big + 4 * (1.45 * big + 16) + 8)
    bound = np.abs(want) * (2 * e + rows * 8 * 2.0 ** -24 + (2.0 ** -20 * big if type_ == "f32" else 0) + 2.0 ** -23) + \
        12 * 2.0 ** -24 * els + 1e-37
    for max_len in (0, 300, 1500, 10 ** 9):
        seqs = s.km.KvSeqs(s.seqs.table, s.seqs.lens, s.seqs.starts, rows=s.rows, max_rows=rows, max_len=max_len)
        w = torch.zeros((s.cache.pages, 1, 64), device="cuda")
        s.km.kv_weigh(s.cache, seqs, q, lse, w)
        assert (np.abs(host(w) - want) <= bound).all(), max_len


@pytest.mark.parametrize("rows", [1, 90])
def test_weigh_and_evict_past_32_bits(rows):
    """Pages behind the first 2^31 bytes of codes: as in a small cache."""
    torch = torch_cuda()
    import paper_2608_14648_amd as km
    heads, page, d = 8, 128, 256  # 256 KiB of codes to a page
    pages = (1 << 31) // (heads * page * d) + 40
    say(f"kv_weigh and kv_evict large: {pages} pages, {rows} rows")
    large, small = km.kv_cache(pages, heads, d, page), km.kv_cache(4, heads, d, page)
    rng = np.random.default_rng(2)
    x, y = (torch.from_numpy(rng.standard_normal((300, heads, d)).astype(np.float32)).bfloat16().cuda() for _ in range(2))
    got = []
    for c, table in ((large, [pages - 1, 5, pages - 7]), (small, [1, 0, 3])):
        t = torch.tensor([table], dtype=torch.int32, device="cuda")
        lens = torch.tensor([300], dtype=torch.int32, device="cuda")
        km.kv_write(c, km.KvSeqs(t, lens, rows=300, max_rows=300), x, y)
        seqs = km.KvSeqs(t, lens, rows=rows, max_rows=rows, max_len=300)
        _, lse = km.kv_attend(c, seqs, x[:rows].contiguous(), lse=True)
        w = torch.zeros((c.pages, heads, page), device="cuda")
        km.kv_weigh(c, seqs, x[:rows].contiguous(), lse, w)
        kept, left = km.kv_evict(c, seqs, w, torch.tensor([140], dtype=torch.int32, device="cuda"), 140, 4, 16)
        back = km.kv_read(c, km.KvSeqs(t, left, rows=140, max_rows=140))
        got.append((kept, left) + back + (w[torch.tensor(table[:2], device="cuda").long()][:, :, :12],))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_evict_long():
    """One long sequence; the order of positions and the digits of the weights."""
    torch = torch_cuda()
    s = Setup4(64, 2, 32, [70001], [1], seed=35)
    w, wd = _weights(s)
    w[:] = np.float32(0.25) * (w * 4).round()  # many ties
    wd.copy_(torch.from_numpy(w))
    _evict(s, w, wd, [30000], 30000, 4, 300, label="long")


@pytest.mark.parametrize("fmt", FMTS)
def test_rotate_write_attend_weigh_evict(fmt):
    """A run of them as a serving program makes it: prompts, single tokens, eviction whenever a sequence is past its budget, rotary
    positions that go on; each step against the oracle, attention over what is left."""
    import oracle.kv_ops as ops
    from test_gpu_kv import _attend_check
    from test_gpu_kv_rotate import _check
    torch = torch_cuda()
    heads, group, d, page, budget = 2, 3, 64, 16, 40
    lens = [50, 7, 33]
    s = _setup(fmt, page, heads, d, [l + 20 for l in lens], lens, seed=71)
    km = s.km
    rot = km.kv_rotary(d)
    freq = 10000.0 ** (-2.0 * np.arange(d // 2) / d)
    w = np.zeros((s.cache.pages, heads, page), np.float32)
    wd = torch.from_numpy(w).cuda()
    s.lens = np.array(lens, np.int32)
    true = np.array(lens)  # tokens seen, evicted ones included
    for step in range(8):
        rows = lens if step == 0 else [1, 1, 1]
        s.starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        s.rows, s.max_rows = int(s.starts[-1]), max(rows)
        s.seqs = s.seqs_of(s.lens, s.starts)
        q, k, v = (s.normal((s.rows, n, d), "bf16") for n in (heads * group, heads, heads))
        pos = np.concatenate([np.arange(t - r, t) for t, r in zip(true, rows)])
        at = torch.from_numpy(pos.astype(np.int32)).cuda()
        q2, k2 = km.kv_rotate(rot, at, q, k)
        _check(q2, q, pos, freq, d, "halves", "bf16")
        _check(k2, k, pos, freq, d, "halves", "bf16")
        s.write(k2, v)
        s.check_cache(f"step {step}")
        _attend_check(s, q2, "bf16", label=f"step {step}")
        _, lse = km.kv_attend(s.cache, s.seqs, q2, lse=True)
        before = host(wd).copy()
        km.kv_weigh(s.cache, s.seqs, q2, lse, wd)
        want, big, els = ops.weigh(s.orc, s.table, s.lens, s.starts, q2.float().cpu().numpy(), host(lse), before,
                                   float(np.float32(1 / math.sqrt(d))))
        e = 2.0 ** -24 * (d * big + 4 * (1.45 * big + 16) + 8)
        room = np.abs(want) * (2 * e + s.max_rows * group * 2.0 ** -24 + 2.0 ** -23) + 12 * 2.0 ** -24 * els
        assert (np.abs(host(wd) - want) <= room).all()
        w = host(wd).copy()
        _, left = _evict(s, w, wd, [budget] * 3, budget, 2, 4, label=f"step {step}")
        s.lens = host(left).astype(np.int32) + 1
        true = true + 1


def test_evict_and_weigh_in_a_graph():
    """Captured on another stream and replayed with new weights and lengths, eager work in between; two graphs side by side."""
    torch = torch_cuda()
    s = Setup4(16, 2, 64, [200, 90], [1, 1], seed=81)
    km = s.km
    q = s.normal((2, 4, 64), "bf16")
    wd = _weights(s)[1]
    keep = torch.tensor([50, 30], dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step():
        _, lse = km.kv_attend(s.cache, s.seqs, q, lse=True)
        km.kv_weigh(s.cache, s.seqs, q, lse, wd)
        return km.kv_evict(s.cache, s.seqs, wd, keep, 50, 2, 3)

    state = (s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale, wd)
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            held = step()
        graphs.append((g, held))
    for i in range(4):
        g, held = graphs[i % 2]
        s.seqs.lens.copy_(torch.tensor([200 - 7 * i, 90 - i], dtype=torch.int32))
        q.copy_(s.normal((2, 4, 64), "bf16"))
        wd.copy_(_weights(s)[1])
        was = [t.clone() for t in state]
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held + state]
        for t, x in zip(state, was):
            t.copy_(x)
        want = step() + state
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_workspace_from_the_pool_and_refusals():
    import ctypes as ct
    torch = torch_cuda()
    from paper_2608_14648_amd import _kv
    from paper_2608_14648_amd._kmq import lib
    s = Setup4(16, 2, 64, [200, 90], [1, 1], seed=91)
    w, wd = _weights(s)
    keep = torch.tensor([50, 30], dtype=torch.int32, device="cuda")
    kept = torch.empty((2, 2, 50), dtype=torch.int32, device="cuda")
    left = torch.empty(2, dtype=torch.int32, device="cuda")
    import oracle.kv_ops as ops
    st = lib().kv_evict(s.cache._ref, s.seqs._ref, wd.data_ptr(), keep.data_ptr(), 50, 0, 0, kept.data_ptr(), left.data_ptr(),
                        None, 0, _kv._raw_stream(0))
    assert st == 0
    torch.cuda.synchronize()
    want, want_left = ops.evict(s.orc, s.table, s.lens, w, [50, 30], 50)
    np.testing.assert_array_equal(host(kept), want)
    np.testing.assert_array_equal(host(left), want_left)
    s.check_cache("pool")
    # the lengths of the call are read by all of its kernels
    assert lib().kv_evict(s.cache._ref, s.seqs._ref, wd.data_ptr(), keep.data_ptr(), 50, 0, 0, kept.data_ptr(),
                          s.seqs.lens.data_ptr(), None, 0, _kv._raw_stream(0)) == -1
    one = s.km.KvSeqs(s.seqs.table[:1].expand(2, -1), s.seqs.lens)
    with pytest.raises(s.km.KmqError, match="share"):
        s.km.kv_evict(s.cache, one, wd, keep, 50)
    q = s.normal((2, 4, 64), "bf16")
    with pytest.raises(s.km.KmqError, match="share"):
        s.km.kv_weigh(s.cache, one, q, torch.zeros((2, 4), device="cuda"), wd)
