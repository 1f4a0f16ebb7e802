"""The key/value cache in 4 bits against the 64-bit oracle (oracle/kv_ops.py).

Codes, scales and the rows read back are compared exactly.  Attention is compared within the bound of test_gpu_kv.py: the outputs'
rounding, the weights', the error of a weight's exponent and of sums; a score's product with its token's scale and the sum with the
scale's logarithm are two more roundings of an exponent's size, within the 4 T of that bound.
"""
import math

import numpy as np
import pytest

from gpu_util import host, say, torch_cuda
from test_gpu_kv import DT, EIGHT, _attend_check
from test_gpu_kv import SPLITS as SPLITS8

pytestmark = pytest.mark.gpu


def _km():
    import paper_2608_14648_amd as km
    return km


class Setup4:
    """A 4-bit cache with garbage in it, on the GPU and in the oracle, and the sequences of a call."""

    def __init__(self, page, heads, d, lens, rows, seed, spare=2, wide=0, spread=0.4):
        import oracle.kv_ops as ops
        import oracle.kv as okv
        torch = torch_cuda()
        km = _km()
        self.torch, self.km, self.fmt = torch, km, "int4"
        self.rng = rng = np.random.default_rng(seed)
        per = [-(-max(l, 0) // page) for l in lens]
        pages = sum(per) + spare
        order = rng.permutation(pages)
        self.table = np.full((len(lens), max(max(per), 1) + wide), -1, np.int32)
        at = 0
        for b, p in enumerate(per):
            self.table[b, :p] = order[at:at + p]
            at += p
        self.lens = np.array(lens, np.int32)
        self.starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.rows, self.max_rows = int(self.starts[-1]), int(max(rows))
        val = rng.integers(-7, 8, (2, pages, heads, page, d))
        wide = np.array([0.4, spread]).reshape(2, 1, 1, 1)  # of keys, of values
        mul = okv.short(np.exp(1.0 + wide * rng.standard_normal((2, pages, heads, page))).astype(np.float32))
        self.orc = ops.Cache4(val[0], np.swapaxes(val[1], 2, 3), mul[0], mul[1])
        k = torch.from_numpy(ops.pack4(val[0])).cuda()
        v = torch.from_numpy(np.ascontiguousarray(ops.pack4(np.swapaxes(val[1], 2, 3)))).cuda()
        sc = torch.from_numpy(np.float32(1.0) / mul).cuda()
        self.cache = km.KvCache(k, v, sc[0].contiguous(), sc[1].contiguous())
        self.seqs = self.seqs_of(self.lens, self.starts)

    def seqs_of(self, lens, starts, table=None):
        torch = self.torch
        t = torch.from_numpy(self.table if table is None else table).cuda()
        return self.km.KvSeqs(t, torch.from_numpy(np.asarray(lens, np.int32)).cuda(),
                              torch.from_numpy(np.asarray(starts, np.int32)).cuda(), rows=int(starts[-1]),
                              max_rows=int(np.diff(starts).max()))

    def normal(self, shape, type_, size=1.0):
        x = self.torch.from_numpy((self.rng.standard_normal(shape) * size).astype(np.float32))
        return x.to(getattr(self.torch, DT[type_])).cuda()

    def check_cache(self, label):
        import oracle.kv_ops as ops
        self.torch.cuda.synchronize()
        for which, name in ((0, "k"), (1, "v")):
            got = ops.unpack4(host((self.cache.k, self.cache.v)[which]))
            got = np.swapaxes(got, 2, 3) if which else got
            np.testing.assert_array_equal(got, self.orc.codes[which], err_msg=f"{label}: {name} codes")
            np.testing.assert_array_equal(host((self.cache.k_scale, self.cache.v_scale)[which]), self.orc.scales(which),
                                          err_msg=f"{label}: {name} scales")

    def write(self, k, v, lens=None, starts=None):
        lens = self.lens if lens is None else lens
        starts = self.starts if starts is None else starts
        self.km.kv_write(self.cache, self.seqs_of(lens, starts), k, v)
        f = [x.float().cpu().numpy().astype(np.float64) for x in (k, v)]
        self.orc.write(self.table, lens, starts, *f)

    def read_check(self, dtype, label):
        """Every row of every sequence back."""
        starts = np.concatenate([[0], np.cumsum(self.lens)])
        gk, gv = self.km.kv_read(self.cache, self.seqs_of(self.lens, starts), dtype)
        self.torch.cuda.synchronize()
        top = self.torch.finfo(dtype).max
        for which, got in ((0, gk), (1, gv)):
            want = np.concatenate([self.orc.rows(self.table[b], 0, ln)[which] for b, ln in enumerate(self.lens)])
            want = self.torch.from_numpy(want.astype(np.float32)).clamp(-top, top).to(dtype)
            np.testing.assert_array_equal(got.float().cpu().numpy(), want.float().numpy(), err_msg=label)


WRITES = [
    # page, heads, d, lens, rows
    (16, 1, 32, [1], [1]),
    (16, 2, 64, [1, 16, 17, 40], [1, 16, 2, 40]),
    (32, 3, 96, [33, 5, 64, 0], [1, 5, 33, 0]),
    (64, 2, 128, [200, 64, 129], [137, 1, 129]),
    (64, 1, 160, [63, 65, 128], [3, 20, 64]),
    (128, 2, 256, [300, 127], [45, 127]),
    (128, 1, 224, [129, 128], [17, 16]),
    (16, 5, 192, [31, 18], [30, 3]),
]


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", range(len(WRITES)))
def test_write_and_read_exact(type_, case):
    page, heads, d, lens, rows = WRITES[case]
    say(f"kv_write int4 {type_} page={page} heads={heads} d={d} lens={lens} rows={rows}")
    s = Setup4(page, heads, d, lens, rows, seed=100 + case)
    shape = (s.rows, heads, d)
    size = np.exp(s.rng.normal(0, 1.5, (s.rows, heads, 1)))
    k, v = s.normal(shape, type_, size), s.normal(shape, type_, size)
    s.write(k, v)
    s.check_cache("write")
    s.read_check(k.dtype, "read")


@pytest.mark.parametrize("type_", ["f32", "bf16"])
def test_write_token_by_token(type_):
    """Neighbouring tokens share bytes of the values: each write leaves the other half as it was."""
    s = Setup4(16, 2, 32, [40, 39], [1, 1], seed=7)
    starts = np.array([0, 1, 2])
    for t in range(1, 40):
        k, v = s.normal((2, 2, 32), type_), s.normal((2, 2, 32), type_, 3.0)
        s.write(k, v, lens=np.array([t + 1, t]), starts=starts)
        s.check_cache(f"token {t}")


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
def test_write_special_values(type_):
    """Zeros, ties, subnormals, the type's largest value, infinities and NaN, past both ends of the scales' range."""
    torch = torch_cuda()
    d = 64
    s = Setup4(16, 1, d, [16] * 8, [16] * 8, seed=11)
    dt = getattr(torch, DT[type_])
    x = s.normal((128, 1, d), type_).cpu()
    top, tiny = torch.finfo(dt).max, torch.finfo(dt).tiny
    x[0:16] = 0.0
    x[16:32] = (torch.arange(d) % 14 * 0.5 + 0.5).to(dt)  # halves of codes for a largest value of 7
    x[17] = -x[16]
    x[32:48] *= tiny
    x[48:64] = top
    x[49] = -top
    x[50, 0, 1:] = 1.0  # beside the largest value
    x[70, 0, 3], x[71, 0, 4], x[72, 0, 5] = math.inf, -math.inf, math.nan
    x[80:96] = math.nan
    x[96:112] = math.inf
    x[97] = 0.0
    x[97, 0, 9] = -math.inf
    x[112:128] = torch.linspace(-7, 7, 16 * d).view(16, 1, d).to(dt)
    x = x.cuda()
    s.write(x, -x)
    s.check_cache("special")
    gk, _ = s.km.kv_read(s.cache, s.seqs, dt)
    assert bool(torch.isfinite(gk.float()).all())


def test_write_at_the_last_bit_of_a_tie():
    """fp32 values a last bit beside code + 1/2: the exact product decides, not the rounded one."""
    torch = torch_cuda()
    s = Setup4(16, 1, 64, [16], [16], seed=3)
    base = np.tile((np.arange(63) % 6 + 0.5).astype(np.float32), (16, 1))
    near = base / np.float32(1.01171875)
    x = np.empty((16, 64), np.float32)
    x[:, 0] = 7.0 / 1.01171875
    pick = np.arange(63) % 3
    x[:, 1:] = np.where(pick == 0, near, np.where(pick == 1, np.nextafter(near, np.float32(1e9)),
                                                  np.nextafter(near, np.float32(0))))
    t = torch.from_numpy(x.reshape(16, 1, 64)).cuda()
    s.write(t, -t)
    s.check_cache("ties")


def test_strided_rows_and_rows_before_the_start():
    torch = torch_cuda()
    heads, d = 2, 64
    s = Setup4(16, heads, d, [20, 3], [4, 5], seed=5)  # two rows of sequence 1 fall before position 0
    fused = s.normal((s.rows, 3 * heads, d), "bf16")
    k, v = fused[:, heads:2 * heads], fused[:, 2 * heads:]
    s.write(k, v)
    s.check_cache("strided")
    buf = torch.full((s.rows, 2 * heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    s.km.kv_read(s.cache, s.seqs, k=buf[:, :heads], v=buf[:, heads:])
    got = buf.float().cpu().numpy()
    assert (got[4:6] == 0).all()
    want = s.orc.rows(s.table[1], 0, 3)
    for which, part in ((0, got[6:9, :heads]), (1, got[6:9, heads:])):
        np.testing.assert_array_equal(part, torch.from_numpy(want[which].astype(np.float32)).bfloat16().float().numpy())


ATTENDS = [
    # page, heads, group, d, lens, rows, window
    (16, 1, 1, 32, [1], [1], 0),
    (16, 2, 1, 64, [1, 15, 16, 17, 63, 64, 65], [1] * 7, 0),
    (16, 2, 4, 64, [100, 257, 31], [1, 1, 1], 0),
    (64, 2, 4, 128, [777, 64, 1, 129], [1] * 4, 0),
    (128, 1, 8, 128, [300, 1025], [1, 1], 0),
    (32, 1, 16, 96, [333, 32], [1, 1], 0),
    (64, 2, 2, 192, [129, 500], [1, 1], 0),
    (64, 1, 4, 256, [65, 400], [1, 1], 0),
    (64, 1, 32, 128, [260], [1], 0),
    (16, 1, 1, 128, [2000], [1], 0),
    (32, 2, 3, 160, [50, 40], [7, 40], 0),
    (16, 1, 2, 224, [33, 64], [33, 20], 0),
    (64, 2, 4, 128, [300, 90], [5, 90], 0),
    (64, 1, 4, 64, [200, 130, 3], [130, 130, 3], 0),
    (64, 1, 4, 32, [90, 130, 3], [70, 1, 3], 0),
    (16, 1, 1, 128, [150], [150], 0),
    (128, 1, 6, 128, [170, 301], [170, 63], 0),
    (32, 1, 2, 128, [100, 400], [3, 70], 33),
    (64, 2, 8, 128, [1000, 70], [4, 4], 64),
    (64, 1, 1, 64, [500], [1], 1),
    (64, 1, 4, 256, [150, 70], [150, 64], 50),
    (16, 1, 4, 96, [150, 70], [150, 64], 0),
]


@pytest.mark.parametrize("type_", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attend(type_, case):
    page, heads, group, d, lens, rows, window = ATTENDS[case]
    say(f"kv_attend int4 {type_} page={page} heads={heads}x{group} d={d} lens={lens} rows={rows} window={window}")
    s = Setup4(page, heads, d, lens, rows, seed=200 + case)
    q = s.normal((s.rows, heads * group, d), type_, 0.6)
    _attend_check(s, q, type_, window=window, label="causal")
    if not window:
        _attend_check(s, q, type_, causal=False, label="whole")


@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("type_", ["bf16", "f32"])
def test_attend_scales_far_apart(rows, type_):
    """Tokens whose value scales lie up to 2^40 apart, side by side."""
    s = Setup4(16, 1, 64, [300, 129], [rows, rows], seed=21, spread=4.0)
    q = s.normal((s.rows, 4, 64), type_, 0.6)
    _attend_check(s, q, type_, label="far apart")


@pytest.mark.parametrize("rows", [1, 70])
def test_attend_both_ends_of_the_scales(rows):
    """Rows of zeros (the least scale, 2^-30) beside values as large as scales get: what the zeros weigh still counts."""
    torch = torch_cuda()
    s = Setup4(16, 1, 64, [200, 90], [rows, rows], seed=23)
    n = int(s.lens.sum())
    k, v = s.normal((n, 1, 64), "f32"), s.normal((n, 1, 64), "f32")
    v[::2] = 0.0
    v[1::6] *= 2.0 ** 30
    v[3::6] *= 2.0 ** -28
    k[5::11] = 0.0
    starts = np.concatenate([[0], np.cumsum(s.lens)])
    s.write(k, v, starts=starts)
    s.check_cache("both ends")
    q = s.normal((s.rows, 4, 64), "bf16")
    _attend_check(s, q, "bf16", label="both ends")


@pytest.mark.parametrize("rows", [1, 70])
def test_attend_rows_that_see_nothing(rows):
    s = Setup4(16, 1, 64, [0, 40, 100, 33], [rows, rows, rows, rows], seed=9, wide=2)
    q = s.normal((s.rows, 4, 64), "bf16")
    _attend_check(s, q, "bf16", label="short")
    table = s.table.copy()
    table[1, :] = -1
    table[2, 1:3] = 10 ** 6
    table[3, 0] = -5
    _attend_check(s, q, "bf16", table=table, label="absent pages")
    _attend_check(s, q, "bf16", table=table, causal=False, label="absent pages, whole")


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("rows", [1, 40, 200])
def test_attend_ignores_what_lies_behind_the_end(page, rows):
    """Codes and scales behind the end of a sequence (NaN, infinite and huge scales) change nothing."""
    torch = torch_cuda()
    s = Setup4(page, 2, 64, [200, 217, 210], [rows, rows, rows], seed=13, wide=5)
    q = s.normal((s.rows, 4, 64), "f16")
    a, la = s.km.kv_attend(s.cache, s.seqs, q, lse=True)
    used = np.zeros((s.cache.pages, page), bool)
    for b, ln in enumerate(s.lens):
        for j in range(ln):
            used[s.table[b, j // page], j % page] = True
    free = torch.from_numpy(~used).cuda()[:, None].expand(s.cache.k_scale.shape)
    for t, x in ((s.cache.k_scale, math.nan), (s.cache.v_scale, math.nan), (s.cache.k_scale, math.inf),
                 (s.cache.v_scale, 1e38), (s.cache.v_scale, 0.0)):
        t[free] = x
        b, lb = s.km.kv_attend(s.cache, s.seqs, q, lse=True)
        assert torch.equal(a, b) and torch.equal(la, lb), x


@pytest.mark.parametrize("rows", [1, 64])
def test_attend_not_finite_queries_stay_in_their_row(rows):
    torch = torch_cuda()
    s = Setup4(64, 2, 128, [300, 200], [rows, rows], seed=31)
    q = s.normal((s.rows, 4, 128), "bf16")
    a, _ = s.km.kv_attend(s.cache, s.seqs, q)
    q2 = q.clone()
    q2[0, 1, 5], q2[s.rows - 1, 2, 7] = math.nan, math.inf
    b, lse = s.km.kv_attend(s.cache, s.seqs, q2, lse=True)
    bad = torch.zeros(a.shape[:2], dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[s.rows - 1, 2] = True
    assert bool(b[bad].isnan().all()) and bool(lse[bad].isnan().all())
    assert torch.equal(a[~bad], b[~bad])


SPLITS = {
    # page, heads, group, d, lens, rows: calls that are split, dealt out, or large in one way
    "one_long": (64, 2, 4, 128, [9000], [1]),
    "one_long_small_pages": (16, 2, 6, 96, [7001], [1]),
    "ragged": (64, 8, 4, 64, [1 + 97 * i % 4001 for i in range(24)], [1] * 24),
    "check": (32, 4, 8, 128, [3000, 2500, 1000, 40], [4, 4, 4, 4]),
    "long_prompt_end": (64, 1, 4, 128, [5000], [40]),
}


@pytest.mark.parametrize("type_", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(SPLITS))
def test_attend_split(name, type_):
    page, heads, group, d, lens, rows = SPLITS[name]
    say(f"kv_attend int4 split {name} {type_}")
    s = Setup4(page, heads, d, lens, rows, seed=41)
    q = s.normal((s.rows, heads * group, d), type_, 0.8)
    _attend_check(s, q, type_, label=name)


# The calls of the 8-bit formats that are split up in one way or another, or take workgroups of eight waves.
CUTS = {n: c for n, c in list(SPLITS8.items()) + [("eight_" + n, c) for n, c in EIGHT.items()] if c[3] % 32 == 0}


@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("name", list(CUTS))
def test_attend_cut_up(name, type_):
    page, heads, group, d, lens, rows, window, wide = CUTS[name]
    say(f"kv_attend int4 cut up {name} {type_}")
    s = Setup4(page, heads, d, lens, rows, seed=700 + list(CUTS).index(name), wide=wide)
    # fp16 results below its normal range are rounded to steps of 2^-24
    _attend_check(s, s.normal((s.rows, heads * group, d), type_, 0.4), type_, window=window, label=name,
                  least=2.0 ** -25 if type_ == "f16" else 0.0)


def test_calls_on_a_stream_and_in_a_graph():
    """write, attend and read captured and replayed with new contents, eager work in between."""
    torch = torch_cuda()
    km = _km()
    s = Setup4(64, 2, 128, [130, 70], [1, 1], seed=51)
    k, v, q = (s.normal((2, h, 128), "bf16") for h in (2, 2, 8))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step():
        km.kv_write(s.cache, s.seqs, k, v)
        return km.kv_attend(s.cache, s.seqs, q, lse=True) + km.kv_read(s.cache, s.seqs)

    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        held = step()
    for i in range(4):
        for t, h in ((k, 2), (v, 2), (q, 8)):
            t.copy_(s.normal((2, h, 128), "bf16"))
        s.seqs.lens.copy_(torch.tensor([130 - i, 70 + i], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_invalid_sequences_are_left_alone():
    torch = torch_cuda()
    s = Setup4(16, 1, 32, [20, 20, 20], [2, 2, 2], seed=61)
    before = [t.clone() for t in (s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale)]
    x = s.normal((6, 1, 32), "bf16")
    for lens, starts in (([-1, 2 ** 30, 33], [0, 2, 4, 6]), ([20, 20, 20], [0, -3, 9, 6])):
        seqs = s.km.KvSeqs(torch.from_numpy(s.table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                           torch.tensor(starts, dtype=torch.int32, device="cuda"), rows=6, max_rows=2)
        s.km.kv_write(s.cache, seqs, x, x)
        out = torch.full_like(x, 5.0)
        s.km.kv_attend(s.cache, seqs, x, out=out)
        k = torch.full_like(x, 5.0)
        s.km.kv_read(s.cache, seqs, k=k, v=torch.empty_like(k))
        torch.cuda.synchronize()
        for t, was in zip((s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale), before):
            assert torch.equal(t, was)
        assert bool((out == 5.0).all()) and bool((k == 5.0).all())


def test_offsets_past_32_bits():
    """Pages behind the first 2^31 bytes of codes and of scales."""
    torch = torch_cuda()
    km = _km()
    heads, page, d = 8, 128, 256  # 128 KiB of codes to a page
    pages = (1 << 31) // (heads * page * d // 2) + 40
    say(f"kv int4 large: {pages} pages")
    cache = km.kv_cache(pages, heads, d, page, torch.uint8)
    small = km.kv_cache(4, heads, d, page, torch.uint8)
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((300, heads, d)).astype(np.float32)).bfloat16().cuda()
    y = torch.from_numpy(rng.standard_normal((300, heads, d)).astype(np.float32)).bfloat16().cuda()
    got = []
    for c, table in ((cache, [pages - 1, 5, pages - 7]), (small, [1, 0, 3])):
        t = torch.tensor([table], dtype=torch.int32, device="cuda")
        seqs = km.KvSeqs(t, torch.tensor([300], dtype=torch.int32, device="cuda"), rows=300, max_rows=300)
        km.kv_write(c, seqs, x, y)
        one = km.KvSeqs(t, torch.tensor([300], dtype=torch.int32, device="cuda"))
        got.append(km.kv_read(c, seqs) + km.kv_attend(c, seqs, x)[:1] + km.kv_attend(c, one, x[:1])[:1])
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_example():
    """The example runs with 4-bit codes.  A code is off by at most half a step of a seventh of the row's largest magnitude, by the
    root of a twelfth of a step on average; of 128 values of a normal distribution the largest is about 2.75 standard deviations (3.6
    in nearly all rows), so keys come back within 3.6 / 7 / sqrt(12) = 15 %."""
    torch = torch_cuda()
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "kv_cache.py")
    spec = importlib.util.spec_from_file_location("kv_cache_example", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    r = ex.main(steps=3, dtype=torch.uint8, say=say)
    assert r["read"] <= 0.15 and math.isfinite(r["prompt"]) and math.isfinite(r["token"])
