"""The 8-bit key/value cache without a GPU: the oracle's definitions against counted-out values, and the refusals of the
C ABI (host checks, before any device call) and of the binding."""
import ctypes as ct
import os

import numpy as np
import pytest

import oracle.kv as okv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_14648_amd", "libkmq.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libkmq.so not built (run __graft_entry__.build())")


def test_e4m3_values_and_rounding():
    v = okv.e4m3_values()
    assert v[0x7E] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1.0 and v[0xB8] == -1.0
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(t[~np.isnan(t)], v[~np.isnan(v)])
    x = np.concatenate([np.linspace(-448, 448, 20011), v[~np.isnan(v)], (v[:126] + v[1:127]) / 2])
    want = torch.from_numpy(x).to(torch.float32)
    x = want.numpy().astype(np.float64)
    np.testing.assert_array_equal(okv.nearest_code(x, "fp8"), want.to(torch.float8_e4m3fn).float().numpy())


def test_multiplier_keeps_eight_bits_and_never_overflows():
    rng = np.random.default_rng(0)
    top = np.exp2(rng.uniform(-140, 127, 20000)).astype(np.float32)
    for fmt, qmax in okv.QMAX.items():
        m = okv.multiplier(top, fmt)
        assert (m.view(np.uint32) & 0xFFFF == 0).all() and (m > 0).all()
        prod = top.astype(np.float64) * m
        assert (prod <= qmax * (1 + 2.0 ** -23)).all()
        assert (prod[m < 2.0 ** 99] >= qmax * (1 - 2.0 ** -7)).all()
        # the scale gives the multiplier back
        s = np.float32(1) / m
        back = okv.short((np.float32(1) / s) * np.float32(1 + 2.0 ** -10))
        np.testing.assert_array_equal(back, m)
    assert okv.multiplier(0.0, "int8") == 2.0 ** 100


def test_oracle_write_by_hand():
    """amax 127 then 254 in a page: the first token's codes halve, ties to even."""
    c = okv.Cache("int8", np.zeros((1, 1, 16, 16)), np.zeros((1, 1, 16, 16)), np.ones((1, 1)), np.ones((1, 1)))
    table = np.array([[0]])
    x = np.arange(-8, 8, dtype=np.float64).reshape(1, 1, 16)
    x[0, 0, 0] = 127
    c.write(table, [1], [0, 1], x, x)
    np.testing.assert_array_equal(c.codes[0][0, 0, 0], x[0, 0])
    assert c.mul[0][0, 0] == 1.0
    y = x.copy()
    y[0, 0, 0] = 254
    c.write(table, [2], [0, 1], y, x)
    assert c.mul[0][0, 0] == 0.5 and c.mul[1][0, 0] == 1.0
    np.testing.assert_array_equal(c.codes[0][0, 0, 0], np.rint(x[0, 0] / 2))
    np.testing.assert_array_equal(c.codes[0][0, 0, 1], np.rint(y[0, 0] / 2))
    np.testing.assert_array_equal(c.codes[1][0, 0, 1], x[0, 0])


def test_oracle_attend_by_hand():
    """Two tokens, one of them twice as likely: the mean weighted 2 : 1."""
    k = np.zeros((1, 1, 16, 16))
    k[0, 0, 0, 0] = 1
    v = np.zeros((1, 1, 16, 16))
    v[0, 0, :, 0], v[0, 0, :, 1] = 3, 6
    c = okv.Cache("int8", k, v, np.ones((1, 1)), np.ones((1, 1)))
    q = np.zeros((2, 1, 16))
    q[:, 0, 0] = np.log(2.0)
    o, lse, *_ = c.attend(np.array([[0]]), [2], [0, 2], q, 1.0)
    np.testing.assert_allclose(o[0, 0], 3.0)
    np.testing.assert_allclose(o[1, 0], 4.0)
    np.testing.assert_allclose(lse[:, 0], [np.log(2.0), np.log(3.0)])
    o, lse, *_ = c.attend(np.array([[0]]), [1], [0, 2], q, 1.0)
    assert (o[0] == 0).all() and np.isneginf(lse[0, 0])


@pytest.fixture(scope="module")
def kmq():
    from paper_2608_14648_amd import _kmq
    return _kmq


def _args(kmq, cache=(), seqs=(), rows=()):
    c = dict(fmt=0, page=64, heads=2, d=128, pages=10, k=0x10000, v=0x20000, k_scale=0x30000, v_scale=0x40000)
    c.update(cache)
    s = dict(n=3, max_pages=4, table=0x50000, table_ld=4, lens=0x60000, starts=None, rows=3, max_rows=1, max_len=0)
    s.update(seqs)
    r = dict(p=0x70000, row=256, head=128)
    r.update(rows)
    return kmq.KmKvCache(**c), kmq.KmKvSeqs(**s), kmq.KmKvRows(**r)


BAD = [
    (dict(fmt=2), {}, {}, -2, "cache format"),
    (dict(page=48), {}, {}, -1, "page ="),
    (dict(page=256), {}, {}, -1, "page ="),
    (dict(d=8), {}, {}, -1, "d ="),
    (dict(d=100), {}, {}, -1, "d ="),
    (dict(d=272), {}, {}, -1, "d ="),
    (dict(heads=0), {}, {}, -1, "heads"),
    (dict(heads=1 << 20), {}, {}, -1, "heads"),
    (dict(pages=0), {}, {}, -1, "pages"),
    (dict(pages=1 << 31), {}, {}, -1, "pages"),
    (dict(k=None), {}, {}, -1, "NULL"),
    (dict(v_scale=None), {}, {}, -1, "NULL"),
    (dict(v=0x20008), {}, {}, -1, "aligned"),
    ({}, dict(n=-1), {}, -1, ">= 0"),
    ({}, dict(max_len=-1), {}, -1, ">= 0"),
    ({}, dict(table=None), {}, -1, "NULL"),
    ({}, dict(lens=None), {}, -1, "NULL"),
    ({}, dict(table_ld=3), {}, -1, "table_ld"),
    ({}, dict(max_pages=0), {}, -1, "max_pages"),
    ({}, dict(max_pages=1 << 26, table_ld=1 << 26), {}, -1, "max_pages"),
    ({}, dict(rows=4), {}, -1, "without starts"),
    ({}, dict(starts=0x80000, rows=1 << 31, max_rows=5), {}, -1, "rows ="),
    ({}, {}, dict(p=None), -1, "NULL"),
    ({}, {}, dict(p=0x70004), -1, "alignment"),
    ({}, {}, dict(row=252), -1, "strides"),
    ({}, {}, dict(head=-128), -1, "strides"),
]


@needs_lib
@pytest.mark.parametrize("cache,seqs,rows,status,msg", BAD)
def test_refusals(kmq, cache, seqs, rows, status, msg):
    L = kmq.lib()
    c, s, r = (ct.byref(x) for x in _args(kmq, cache, seqs, rows))
    good = ct.byref(_args(kmq)[2])
    for st in (L.kv_write(c, s, r, good, 1, None), L.kv_write(c, s, good, r, 1, None) if rows else status,
               L.kv_read(c, s, r, good, 1, None),
               L.kv_attend(c, s, r, 4, 0.1, 1, 0, good, 1, None, None, 0, None)):
        assert st == status
    assert msg in L.km_last_error().decode()
    if not rows:
        assert L.kv_attend_bytes(c, s, 4, 1, 0, 1) == status


@needs_lib
def test_attend_refusals_and_empty_calls(kmq):
    L = kmq.lib()
    c, s, r = (ct.byref(x) for x in _args(kmq))

    def call(q_heads=4, scale=0.1, flags=1, window=0, type_=1, lse=None, ws=None, ws_bytes=0, seqs=s):
        return L.kv_attend(c, seqs, r, q_heads, scale, flags, window, r, type_, lse, ws, ws_bytes, None)

    for kw, status, msg in [
        (dict(q_heads=3), -1, "q_heads"), (dict(q_heads=0), -1, "q_heads"), (dict(scale=0.0), -1, "scale"),
        (dict(scale=-1.0), -1, "scale"), (dict(scale=float("nan")), -1, "scale"), (dict(scale=float("inf")), -1, "scale"),
        (dict(flags=2), -1, "flags"), (dict(window=-1), -1, "window"), (dict(flags=0, window=5), -1, "window"),
        (dict(type_=3), -2, "type"),
    ]:
        assert call(**kw) == status, kw
        assert msg in L.km_last_error().decode(), kw
    # a workspace that is too small or not aligned; a long table of one sequence is split
    big = _args(kmq, seqs=dict(n=1, rows=1, max_pages=1000, table_ld=1000))[1]
    need = L.kv_attend_bytes(c, ct.byref(big), 4, 1, 0, 1)
    assert need > 0
    for ws, nb in ((0x90000, need - 1), (0x90008, need)):
        assert call(ws=ws, ws_bytes=nb, seqs=ct.byref(big)) == -1
        assert "ws" in L.km_last_error().decode()
    assert L.kv_write(c, s, r, r, 7, None) == -2
    assert L.kv_read(None, s, r, r, 1, None) == -1
    assert L.kv_read(c, None, r, r, 1, None) == -1
    # nothing to do: OK without a device
    none = _args(kmq, seqs=dict(n=0, rows=0, max_rows=0, table=None, lens=None))[1]
    assert L.kv_write(c, ct.byref(none), None, None, 1, None) == 0
    assert call(seqs=ct.byref(none)) == 0
    assert L.kv_attend_bytes(c, ct.byref(none), 4, 1, 0, 1) == 0


@needs_lib
def test_binding_refuses_host_tensors():
    import torch
    import paper_2608_14648_amd as km
    z = torch.zeros((1, 1, 16, 16), dtype=torch.int8)
    with pytest.raises(ValueError):
        km.KvCache(z, z, torch.ones(1, 1), torch.ones(1, 1))
    with pytest.raises(TypeError):
        km.KvCache(z.float(), z, torch.ones(1, 1), torch.ones(1, 1))
    with pytest.raises(TypeError):
        km.kv_cache(1, 1, 16, dtype=torch.float32, device="cpu")
    with pytest.raises(ValueError):
        km.KvSeqs(torch.zeros((1, 1), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


@needs_lib
def test_table_rows_of_one_address_or_apart(kmq):
    """The stride of the descriptor is the table's own: 0 for one row expanded to all sequences; rows that overlap in part are
    refused.  (Fake tensors: shapes and strides without memory.)"""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    import paper_2608_14648_amd as km
    with FakeTensorMode():
        def table(n, width, row):
            return torch.empty(n * max(row, 1) + width, dtype=torch.int32, device="cuda:0").as_strided((n, width), (row, 1))
        lens = torch.empty(3, dtype=torch.int32, device="cuda:0")
        for row, ld in ((0, 0), (5, 5), (8, 8)):
            assert km.KvSeqs(table(3, 5, row), lens)._c.table_ld == ld
        for row in (1, 4):
            with pytest.raises(ValueError, match="overlap"):
                km.KvSeqs(table(3, 5, row), lens)
        assert km.KvSeqs(table(1, 5, 0), lens[:1])._c.table_ld == 5
    c, s, _ = (ct.byref(x) for x in _args(kmq, seqs=dict(table_ld=0)))
    assert kmq.lib().kv_attend_bytes(c, s, 4, 1, 0, 1) == 0


@needs_lib
def test_plan_of_the_largest_calls(kmq):
    """Tables of 2^30 positions with many row tiles: the chunks of all tiles pass 2^40 and their share per workgroup 2^31."""
    L = kmq.lib()
    for heads, n, rows in ((8, 128, 8192), (8, 128, 8191), (8, 100, 20000), (1, 2000, 70000)):
        c, s, _ = (ct.byref(x) for x in _args(kmq, dict(heads=heads), dict(n=n, max_pages=1 << 24, table_ld=1 << 24,
                                                                           max_rows=rows, rows=n * rows)))
        # tiles enough for the whole card: none is split, no workspace
        assert L.kv_attend_bytes(c, s, 2 * heads, 1, 0, 1) == 0, L.km_last_error().decode()


@needs_lib
def test_binding_refuses_tensors_of_several_devices():
    """Every tensor of a cache and of the sequences is on one GPU.  (Fake tensors: no memory, so two GPUs are not needed.)"""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    import paper_2608_14648_amd as km
    with FakeTensorMode():
        def codes(dev):
            return torch.empty((2, 1, 16, 16), dtype=torch.int8, device=dev)

        def scales(dev):
            return torch.empty((2, 1), device=dev)

        def ints(n, dev):
            return torch.empty(n, dtype=torch.int32, device=dev)

        a, b = "cuda:0", "cuda:1"
        km.KvCache(codes(a), codes(a), scales(a), scales(a))
        for devs, name in (((a, b, a, a), "v"), ((a, a, b, a), "k_scale"), ((b, b, b, a), "v_scale")):
            with pytest.raises(ValueError, match=f"^{name} must be on"):
                km.KvCache(codes(devs[0]), codes(devs[1]), scales(devs[2]), scales(devs[3]))
        table = torch.empty((3, 4), dtype=torch.int32, device=a)
        km.KvSeqs(table, ints(3, a), ints(4, a), rows=9)
        with pytest.raises(ValueError, match="^lens must be on"):
            km.KvSeqs(table, ints(3, b))
        with pytest.raises(ValueError, match="^starts must be on"):
            km.KvSeqs(table, ints(3, a), ints(4, b), rows=9)


@needs_lib
def test_binding_refuses_rows_that_require_grad():
    """No result without its graph: refused while gradients are recorded, taken where they are off.  (Fake tensors; without rows
    there is nothing to launch.)"""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    import paper_2608_14648_amd as km
    with FakeTensorMode():
        dev = "cuda:0"
        codes, scales = torch.empty((2, 1, 16, 16), dtype=torch.int8, device=dev), torch.empty((2, 1), device=dev)
        cache = km.KvCache(codes, codes, scales, scales)
        none = torch.empty(0, dtype=torch.int32, device=dev)
        seqs = km.KvSeqs(torch.empty((0, 1), dtype=torch.int32, device=dev), none)
        x = torch.empty((0, 1, 16), device=dev)
        g = torch.empty((0, 1, 16), device=dev, requires_grad=True)
        calls = [lambda t: km.kv_write(cache, seqs, t, x), lambda t: km.kv_write(cache, seqs, x, t),
                 lambda t: km.kv_read(cache, seqs, k=t, v=x), lambda t: km.kv_attend(cache, seqs, t),
                 lambda t: km.kv_attend(cache, seqs, x, out=t)]
        for call in calls:
            with pytest.raises(ValueError, match="requires grad"):
                call(g)
            call(x)
            call(g.detach())
            with torch.no_grad():
                call(g)


@needs_lib
def test_binding_does_not_wrap_numbers():
    """max_rows, max_len and window past 32 bits: the largest number or a refusal, not their low halves."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    import paper_2608_14648_amd as km
    from paper_2608_14648_amd import _kv
    seen = []

    class Lib:
        def kv_attend_bytes(self, cache, seqs, q_heads, flags, window, type_):
            seen.append(window)
            return -1

        def km_last_error(self):
            return b"seen"

    with FakeTensorMode():
        dev = "cuda:0"
        codes, scales = torch.empty((2, 1, 16, 16), dtype=torch.int8, device=dev), torch.empty((2, 1), device=dev)
        cache = km.KvCache(codes, codes, scales, scales)
        table = torch.empty((2, 4), dtype=torch.int32, device=dev)
        lens, starts = (torch.empty(n, dtype=torch.int32, device=dev) for n in (2, 3))
        top = 2 ** 31 - 1
        for given, held in ((2 ** 32 + 1, top), (2 ** 31, top), (top, top), (7, 7), (-2 ** 32 + 5, -1)):
            s = km.KvSeqs(table, lens, starts, rows=5, max_rows=given, max_len=given)
            assert (s._c.max_rows, s._c.max_len) == (held, held)
            with pytest.MonkeyPatch.context() as m:
                m.setattr(_kv, "lib", Lib)
                with pytest.raises(km.KmqError, match="seen"):
                    km.kv_attend(cache, s, torch.empty((5, 1, 16), device=dev), window=given)
            assert seen[-1] == held


@needs_lib
def test_one_sequence_of_more_rows_than_a_grid_takes(kmq):
    """fp32 rows of one sequence, 2^28 of them over the query heads and more, are refused; bf16 ones are launched in pieces."""
    L = kmq.lib()
    for rows, status in (((1 << 24) - 1024, 0), (1 << 24, -1)):
        c, s, _ = (ct.byref(x) for x in _args(kmq, dict(heads=8), dict(n=1, max_pages=1 << 20, table_ld=1 << 20, max_rows=rows,
                                                                     rows=rows)))
        assert L.kv_attend_bytes(c, s, 16, 1, 0, 1) == 0
        assert L.kv_attend_bytes(c, s, 16, 1, 0, 0) == status
    assert "max_rows" in L.km_last_error().decode()


@needs_lib
def test_table_of_one_page_has_any_column_stride():
    """The stride of an axis of one is of no meaning: a row of pages turned into a table of one page each is taken."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    import paper_2608_14648_amd as km
    with FakeTensorMode():
        lens = torch.empty(5, dtype=torch.int32, device="cuda:0")
        table = torch.empty((1, 5), dtype=torch.int32, device="cuda:0").t()
        assert table.stride() == (1, 5) and km.KvSeqs(table, lens)._c.table_ld == 1
        with pytest.raises(ValueError, match="contiguous rows"):
            km.KvSeqs(torch.empty((2, 5), dtype=torch.int32, device="cuda:0").t(), lens)
