"""The 4-bit cache, rotary positions, weights and eviction without a GPU: the oracle's definitions against counted-out values, and the
refusals of the C ABI (host checks, before any device call) and of the binding."""
import ctypes as ct
import math
import os

import numpy as np
import pytest

import oracle.kv as okv
import oracle.kv_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_14648_amd", "libkmq.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libkmq.so not built (run __graft_entry__.build())")


# ---- the oracle ----------------------------------------------------------------------------------------------------

def test_multiplier_of_4_bits():
    rng = np.random.default_rng(0)
    top = np.exp2(rng.uniform(-140, 127, 20000)).astype(np.float32)
    m = ops.multiplier4(top)
    assert (m.view(np.uint32) & 0xFFFF == 0).all() and m.min() == 2.0 ** -30 and m.max() == 2.0 ** 30
    inside = (m > 2.0 ** -30) & (m < 2.0 ** 30)
    prod = top.astype(np.float64) * m
    assert (prod[inside] <= 7 * (1 + 2.0 ** -23)).all() and (prod[inside] >= 7 * (1 - 2.0 ** -7)).all()
    assert ops.multiplier4(0.0) == 2.0 ** 30


def test_pack_and_unpack():
    x = np.arange(-7, 8).repeat(2)[:28].reshape(2, 14).astype(np.float64)
    assert (ops.unpack4(ops.pack4(x)) == x).all()
    assert ops.pack4(np.array([-7.0, 7.0]))[0] == 0xF1  # the first in the low half


def _cache4(pages=1, heads=1, page=16, d=32):
    z = np.zeros((pages, heads, page, d))
    one = np.ones((pages, heads, page))
    return ops.Cache4(z, np.swapaxes(z, 2, 3), one, one)


def test_oracle_write4_by_hand():
    c = _cache4()
    x = np.zeros((2, 1, 32))
    x[0, 0, :15] = np.arange(-7, 8)
    x[1, 0, :4] = [14, 1, 3, -1]  # multiplier 1/2: 0.5 and 1.5 are ties, to 0 and 2
    c.write(np.array([[0]]), [2], [0, 2], x, -x)
    np.testing.assert_array_equal(c.codes[0][0, 0, 0], x[0, 0])
    np.testing.assert_array_equal(c.codes[0][0, 0, 1, :4], [7, 0, 2, 0])
    np.testing.assert_array_equal(c.codes[1][0, 0, 1, :4], [-7, 0, -2, 0])
    assert c.mul[0][0, 0, 0] == 1.0 and c.mul[0][0, 0, 1] == 0.5
    k, v = c.rows(np.array([0]), 1, 2)
    np.testing.assert_array_equal(k[0, 0, :4], [14, 0, 4, 0])


def test_oracle_attend4_by_hand():
    c = _cache4()
    c.codes[0][0, 0, 0, 0] = 1
    c.codes[1][0, 0, 0], c.codes[1][0, 0, 1] = 3, 6
    q = np.zeros((2, 1, 32))
    q[:, 0, 0] = np.log(2.0)
    o, lse, *_ = c.attend(np.array([[0]]), [2], [0, 2], q, 1.0)
    np.testing.assert_allclose(o[0, 0], 3.0)
    np.testing.assert_allclose(o[1, 0], 4.0)
    np.testing.assert_allclose(lse[:, 0], [np.log(2.0), np.log(3.0)])
    # the same as one page per token of the other oracle
    rng = np.random.default_rng(1)
    val = rng.integers(-7, 8, (2, 3, 2, 16, 32))
    mul = okv.short(np.exp(rng.standard_normal((2, 3, 2, 16))).astype(np.float32))
    a = ops.Cache4(val[0], np.swapaxes(val[1], 2, 3), mul[0], mul[1])
    flat = [np.moveaxis(x, 2, 1).reshape(48, 2, 1, 32) for x in val]
    b = okv.Cache("int8", flat[0], np.swapaxes(flat[1], 2, 3), *(np.moveaxis(m, 2, 1).reshape(48, 2) for m in mul))
    q = rng.standard_normal((9, 4, 32))
    table = np.array([[2, 0, 1]])
    wide = (table[..., None] * 16 + np.arange(16)).reshape(1, 48)
    for kw in (dict(), dict(causal=False), dict(window=5)):
        x, y = a.attend(table, [41], [0, 9], q, 0.3, **kw), b.attend(wide, [41], [0, 9], q, 0.3, **kw)
        for m, n in zip(x[:4], y[:4]):
            np.testing.assert_allclose(m, n, rtol=1e-12, atol=1e-12)


def test_oracle_rotate_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    f = [math.pi / 2, math.pi]
    np.testing.assert_allclose(ops.rotate(x, [1], f, 4, "halves")[0, 0], [-3, -2, 1, -4, 9], atol=1e-12)
    np.testing.assert_allclose(ops.rotate(x, [1], f, 4, "pairs")[0, 0], [-2, 1, -3, -4, 9], atol=1e-12)
    np.testing.assert_allclose(ops.rotate(x, [1], f, 4, "halves", inverse=True)[0, 0], [3, -2, -1, -4, 9], atol=1e-12)
    np.testing.assert_allclose(ops.rotate(x, [2], f, 4, "halves", amplitude=2.0)[0, 0], [-2, 4, -6, 8, 9], atol=1e-12)
    # scores depend on differences of positions alone
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 8))
    g = 10.0 ** -np.arange(4)
    a = (ops.rotate(q, [70], g, 8, "pairs") * ops.rotate(k, [61], g, 8, "pairs")).sum()
    b = (ops.rotate(q, [9], g, 8, "pairs") * k).sum()
    assert abs(a - b) < 1e-12


def test_oracle_weigh_by_hand():
    """Two tokens and a row that sees both, one twice as likely."""
    c = _cache4()
    c.codes[0][0, 0, 0, 0] = 1
    q = np.zeros((1, 2, 32))
    q[0, 0, 0] = np.log(2.0)
    w = np.full((1, 1, 16), 5.0)
    lse = np.array([[np.log(3.0), np.log(2.0)]])
    out, *_ = ops.weigh(c, np.array([[0]]), [2], [0, 1], q, lse, w, 1.0, decay=0.5)
    np.testing.assert_allclose(out[0, 0, :3], [2.5 + 2 / 3 + 1 / 2, 1 / 3 + 1 / 2, 5.0])  # the row's own token begins anew
    out, *_ = ops.weigh(c, np.array([[0]]), [2], [0, 1], q, np.array([[-np.inf, np.log(2.0)]]), w, 1.0, decay=0.0)
    np.testing.assert_allclose(out[0, 0, :2], [0.5, 0.5])


def test_oracle_evict_by_hand():
    c = okv.Cache("int8", np.zeros((2, 1, 16, 16)), np.zeros((2, 1, 16, 16)), np.array([[1.0], [0.5]]), np.array([[0.5], [0.5]]))
    for j in range(20):
        c.codes[0][j // 16, 0, j % 16] = j
        c.codes[1][j // 16, 0, j % 16] = -j
    w = np.zeros((2, 1, 16))
    w[0, 0, [2, 9, 11]] = [3, 7, 3]
    w[1, 0, 0] = 5
    kept, left = ops.evict(c, [[0, 1]], [20], w, [5], 6, first=1, recent=1)
    # 0 and 19 always, then 9, 16 and of the equal 2 and 11 the lower
    assert kept[0, 0].tolist() == [0, 2, 9, 16, 19, -1] and left[0] == 5
    assert c.mul[0][0, 0] == 0.5 and c.mul[1][0, 0] == 0.5
    # keys of the first page take the second's multiplier: half the codes, ties to even (0, 1, 4.5 -> 4)
    assert c.codes[0][0, 0, :5, 0].tolist() == [0, 1, 4, 16, 19]
    assert c.codes[1][0, 0, :5, 0].tolist() == [0, -2, -9, -16, -19]
    assert w[0, 0, :5].tolist() == [0, 3, 7, 5, 0]
    assert c.codes[0][0, 0, 5, 0] == 5  # what lies behind stays


# ---- refusals ------------------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def kmq():
    from paper_2608_14648_amd import _kmq
    return _kmq


FAKE = 0x10000


def _args(kmq, cache=(), seqs=(), rows=()):
    c = dict(fmt=4, page=64, heads=2, d=128, pages=10, k=0x10000, v=0x20000, k_scale=0x30000, v_scale=0x40000)
    c.update(cache)
    s = dict(n=3, max_pages=4, table=0x50000, table_ld=4, lens=0x60000, starts=None, rows=3, max_rows=1, max_len=0)
    s.update(seqs)
    r = dict(p=0x70000, row=256, head=128)
    r.update(rows)
    return kmq.KmKvCache(**c), kmq.KmKvSeqs(**s), kmq.KmKvRows(**r)


@needs_lib
def test_four_bits_want_multiples_of_32(kmq):
    L = kmq.lib()
    for d in (16, 48, 80, 240):
        c, s, r = (ct.byref(x) for x in _args(kmq, dict(d=d)))
        for st in (L.kv_write(c, s, r, r, 1, None), L.kv_read(c, s, r, r, 1, None),
                   L.kv_attend(c, s, r, 4, 0.1, 1, 0, r, 1, None, None, 0, None), L.kv_attend_bytes(c, s, 4, 1, 0, 1),
                   L.kv_weigh(c, s, r, 4, 0.1, 1, 0, 1, FAKE, FAKE, 1.0, None, 0, None), L.kv_weigh_bytes(c, s, 4, 1, 0, 1), L.kv_evict_bytes(c, s, 5)):
            assert st == -1 and "multiple of 32" in L.km_last_error().decode()
    for d in (32, 96, 256):
        c, s, r = (ct.byref(x) for x in _args(kmq, dict(d=d)))
        assert L.kv_evict_bytes(c, s, 5) > 0
    for fmt in (2, 3, 5, -1):
        c = ct.byref(_args(kmq, dict(fmt=fmt))[0])
        assert L.kv_write(c, s, r, r, 1, None) == -2 and "cache format" in L.km_last_error().decode()


@needs_lib
def test_rotate_refusals(kmq):
    L = kmq.lib()
    _, s, r = _args(kmq)
    base = dict(dims=64, layout=0, freq=FAKE, amplitude=1.0)

    def call(rot=(), seqs=s, positions=None, rows=0, q=r, hq=4, k=r, hk=2, qo=r, ko=r, d=128, type_=1, flags=0):
        rt = None if rot is None else ct.byref(kmq.KmKvRotary(**{**base, **dict(rot)}))
        p = [None if x is None else ct.byref(x) for x in (seqs, q, k, qo, ko)]
        return L.kv_rotate(rt, p[0], positions, rows, p[1], hq, p[2], hk, p[3], p[4], d, type_, flags, None)

    odd = kmq.KmKvRows(p=0x70004, row=256, head=128)
    for kw, status, msg in [
        (dict(rot=None), -1, "NULL"), (dict(rot=dict(dims=63)), -1, "dims"), (dict(rot=dict(dims=0)), -1, "dims"),
        (dict(rot=dict(dims=130)), -1, "dims"), (dict(rot=dict(layout=2)), -2, "layout"), (dict(rot=dict(freq=None)), -1, "freq"),
        (dict(rot=dict(freq=FAKE + 4)), -1, "freq"), (dict(rot=dict(amplitude=float("nan"))), -1, "amplitude"),
        (dict(flags=2), -1, "flags"), (dict(seqs=None), -1, "either"), (dict(positions=FAKE), -1, "either"),
        (dict(hq=0), -1, "q_heads"), (dict(hk=-1), -1, "k_heads"), (dict(hq=1 << 20), -1, "q_heads"), (dict(d=8), -1, "d ="),
        (dict(d=264), -1, "d ="), (dict(type_=3), -2, "type"), (dict(q=None), -1, "q is NULL"), (dict(qo=None), -1, "q_out is NULL"),
        (dict(k=None), -1, "k is NULL"), (dict(ko=None), -1, "k_out is NULL"), (dict(q=odd), -1, "alignment"),
        (dict(ko=odd), -1, "alignment"), (dict(seqs=None, positions=FAKE, rows=1 << 31), -1, "rows ="),
        (dict(seqs=None, positions=FAKE, rows=-1), -1, "rows ="),
        (dict(seqs=_args(kmq, seqs=dict(rows=4))[1]), -1, "without starts"),
        (dict(seqs=_args(kmq, seqs=dict(lens=None))[1]), -1, "NULL"),
    ]:
        assert call(**kw) == status, kw
        assert msg in L.km_last_error().decode(), (kw, L.km_last_error())
    # nothing to do
    assert call(seqs=_args(kmq, seqs=dict(n=0, rows=0, max_rows=0, table=None, lens=None))[1]) == 0
    assert call(seqs=None, positions=FAKE, rows=0) == 0


@needs_lib
def test_weigh_refusals(kmq):
    L = kmq.lib()
    c, s, r = _args(kmq)

    def call(cache=c, seqs=s, q=r, hq=4, scale=0.1, flags=1, window=0, type_=1, lse=FAKE, weight=FAKE, decay=1.0, ws=None, n=0):
        p = [None if x is None else ct.byref(x) for x in (cache, seqs, q)]
        return L.kv_weigh(p[0], p[1], p[2], hq, scale, flags, window, type_, lse, weight, decay, ws, n, None)

    prompt = _args(kmq, seqs=dict(n=1, max_rows=2000, rows=2000, max_pages=40, table_ld=40))[1]
    need = L.kv_weigh_bytes(ct.byref(c), ct.byref(prompt), 4, 1, 0, 1)
    assert need > 0 and L.kv_weigh_bytes(ct.byref(c), ct.byref(s), 4, 1, 0, 1) == 0

    for kw, status, msg in [
        (dict(cache=None), -1, "NULL"), (dict(seqs=None), -1, "NULL"), (dict(q=None), -1, "q is NULL"), (dict(lse=None), -1, "NULL"),
        (dict(weight=None), -1, "NULL"), (dict(hq=3), -1, "q_heads"), (dict(scale=0.0), -1, "scale"),
        (dict(scale=float("inf")), -1, "scale"), (dict(decay=-1.0), -1, "decay"), (dict(decay=float("nan")), -1, "decay"),
        (dict(decay=float("inf")), -1, "decay"), (dict(flags=2), -1, "flags"), (dict(window=-1), -1, "window"),
        (dict(flags=0, window=4), -1, "window"), (dict(type_=9), -2, "type"),
        (dict(seqs=_args(kmq, seqs=dict(table_ld=0))[1]), -1, "share"),
        (dict(seqs=prompt, ws=FAKE, n=need - 1), -1, "ws"), (dict(seqs=prompt, ws=FAKE + 8, n=need), -1, "ws"),
        (dict(seqs=_args(kmq, seqs=dict(n=1 << 20, rows=1 << 20))[1]), -1, "n * heads"),
        (dict(cache=_args(kmq, dict(k_scale=0x30004))[0]), -1, "scales"),
        (dict(seqs=_args(kmq, seqs=dict(n=1, max_rows=1 << 28, rows=1 << 28, table_ld=0))[1], hq=8), -1, "2^30"),
    ]:
        assert call(**kw) == status, kw
        assert msg in L.km_last_error().decode(), (kw, L.km_last_error())
    assert call(seqs=_args(kmq, seqs=dict(n=0, rows=0, max_rows=0, table=None, lens=None))[1]) == 0


@needs_lib
def test_evict_refusals(kmq):
    L = kmq.lib()
    c, s, _ = _args(kmq)

    def call(cache=c, seqs=s, weight=FAKE, keep=FAKE, max_keep=100, first=0, recent=0, kept=FAKE, lens=FAKE, ws=None, n=0):
        p = [None if x is None else ct.byref(x) for x in (cache, seqs)]
        return L.kv_evict(p[0], p[1], weight, keep, max_keep, first, recent, kept, lens, ws, n, None)

    need = L.kv_evict_bytes(ct.byref(c), ct.byref(s), 100)
    assert need > 0
    for kw, status, msg in [
        (dict(cache=None), -1, "NULL"), (dict(seqs=None), -1, "NULL"), (dict(weight=None), -1, "NULL"), (dict(keep=None), -1, "NULL"),
        (dict(kept=None), -1, "NULL"), (dict(lens=None), -1, "NULL"), (dict(weight=FAKE + 8), -1, "aligned"),
        (dict(lens=0x60000), -1, "sequences' own"), (dict(max_keep=0), -1, "max_keep"), (dict(max_keep=(1 << 30) + 1), -1, "max_keep"),
        (dict(first=-1), -1, "first"), (dict(recent=-1), -1, "recent"), (dict(first=60, recent=41), -1, "together"),
        (dict(ws=FAKE, n=need - 1), -1, "ws"), (dict(ws=FAKE + 8, n=need), -1, "ws"),
        (dict(seqs=_args(kmq, seqs=dict(table_ld=0))[1]), -1, "share"),
        (dict(seqs=_args(kmq, seqs=dict(n=1 << 22))[1]), -1, "n * heads"),
    ]:
        assert call(**kw) == status, kw
        assert msg in L.km_last_error().decode(), (kw, L.km_last_error())
    # the rows of the call play no part
    assert L.kv_evict_bytes(ct.byref(c), ct.byref(_args(kmq, seqs=dict(rows=0, max_rows=0))[1]), 100) == need
    assert call(seqs=_args(kmq, seqs=dict(n=0, rows=0, max_rows=0, table=None, lens=None))[1]) == 0
    for fmt, d in ((0, 128), (1, 80)):
        assert L.kv_evict_bytes(ct.byref(_args(kmq, dict(fmt=fmt, d=d))[0]), ct.byref(s), 100) > 0


def _fake():
    torch = pytest.importorskip("torch")
    from torch._subclasses.fake_tensor import FakeTensorMode
    return torch, FakeTensorMode()


@needs_lib
def test_binding_of_the_4_bit_cache():
    import paper_2608_14648_amd as km
    torch, mode = _fake()
    with mode:
        def t(*shape, dtype=torch.uint8):
            return torch.empty(shape, dtype=dtype, device="cuda:0")
        sc = t(3, 2, 16, dtype=torch.float32)
        c = km.KvCache(t(3, 2, 16, 32), t(3, 2, 64, 8), sc, sc)
        assert (c.pages, c.heads, c.page, c.d, c._c.fmt) == (3, 2, 16, 64, 4)
        for args in ((t(3, 2, 16, 32), t(3, 2, 64, 16), sc, sc), (t(3, 2, 16, 32), t(3, 2, 32, 8), sc, sc),
                     (t(3, 2, 16, 32), t(3, 2, 64, 8), t(3, 2, dtype=torch.float32), sc),
                     (t(3, 2, 16, 32), t(3, 2, 64, 8), sc, t(3, 2, 8, dtype=torch.float32))):
            with pytest.raises(ValueError):
                km.KvCache(*args)
        n = km.kv_cache(3, 2, 64, 16, torch.uint8, device="cuda:0")
        assert tuple(n.k.shape) == (3, 2, 16, 32) and tuple(n.v.shape) == (3, 2, 64, 8) and tuple(n.v_scale.shape) == (3, 2, 16)
        with pytest.raises(ValueError, match="even"):
            km.kv_cache(3, 2, 63, 16, torch.uint8, device="cuda:0")


@needs_lib
def test_binding_refuses_for_rotate():
    import paper_2608_14648_amd as km
    torch, mode = _fake()
    with pytest.raises(ValueError, match="GPU"):
        km.KvRotary(torch.ones(4, dtype=torch.float64))
    for kw, msg in ((dict(dims=3), "even"), (dict(dims=0), "even"), (dict(dims=4, base=0.0), "base"), (dict(dims=4, factor=-1.0), "factor"),
                    (dict(dims=4, scaling="x"), "scaling"), (dict(dims=4, scaling="parts"), "original"),
                    (dict(dims=4, scaling="parts", original=9, low=2.0, high=2.0), "original"), (dict(dims=2, scaling="base"), "pair")):
        with pytest.raises(ValueError, match=msg):
            km.kv_rotary(device="cpu", **kw)
    with mode:
        dev = "cuda:0"
        rot = km.KvRotary(torch.empty(8, dtype=torch.float64, device=dev))
        at = torch.empty(5, dtype=torch.int32, device=dev)

        def rows(n=5, heads=2, d=32, dtype=torch.bfloat16, device=dev, **kw):
            return torch.empty((n, heads, d), dtype=dtype, device=device, **kw)

        def refused(err, msg, *a, **kw):
            with pytest.raises(err, match=msg):
                km.kv_rotate(rot, *a, **kw)

        with pytest.raises(ValueError, match="layout"):
            km.KvRotary(torch.empty(8, dtype=torch.float64, device=dev), "other")
        with pytest.raises(TypeError):
            km.KvRotary(torch.empty(8, device=dev))
        refused(ValueError, "positions", torch.empty(5, dtype=torch.int32), rows())
        refused(TypeError, "positions", at.long(), rows())
        refused(ValueError, "rotary on", torch.empty(5, dtype=torch.int32, device="cuda:1"), rows(device="cuda:1"))
        refused(ValueError, "q must be on", at, rows(device="cuda:1"))
        refused(ValueError, "q must be", at, rows(4))
        refused(ValueError, "k must be", at, rows(), rows(6))
        refused(ValueError, "k must be", at, rows(), rows(d=16))
        refused(TypeError, "k must be", at, rows(), rows(dtype=torch.float16))
        refused(TypeError, "q must be", at, rows(dtype=torch.float64))
        refused(ValueError, "q must be a tensor", at, torch.empty((5, 64), device=dev))
        refused(ValueError, "k_out without k", at, rows(), k_out=rows())
        refused(ValueError, "requires grad", at, rows(requires_grad=True))
        refused(ValueError, "q_out must be", at, rows(), q_out=rows(heads=3))
        refused(ValueError, "contiguous", at, rows(d=64)[..., ::2])
        refused(ValueError, "must not overlap", at, rows(), q_out=rows(1).expand(5, 2, 32))


@needs_lib
def test_rotated_rows_must_not_overlap_others(kmq):
    """In place, or apart: what lies side by side in the same rows is apart.  (On the CPU: the rule looks at addresses alone.)"""
    import torch
    from paper_2608_14648_amd._kv import _apart
    buf = torch.empty((6, 10, 16))
    q, k, v = buf[:, :5], buf[:, 5:8], buf[:, 8:]
    assert _apart(q, k) and _apart(k, q) and _apart(q, v) and _apart(v, k)
    assert not _apart(q, buf[:, 4:6]) and not _apart(buf[:, 4:6], q) and not _apart(q, q) and not _apart(buf, k)
    assert not _apart(buf[1:, :5], buf[:5, :5])  # a row further
    assert _apart(buf[1:, :5], buf[:5, 5:8]) and _apart(buf[:3], buf[3:])
    assert not _apart(buf[:, :5], buf.view(-1)[:6 * 5 * 16].view(6, 5, 16))  # other strides in the same range
    assert not _apart(buf[:1], buf[:1, 2:4]) and _apart(buf[:1, :2], buf[:1, 2:4])
    # the last row of one reaches into the range of the other's last: rows of one stride that are shifted by part of a row
    flat = torch.empty(400)
    a, b = flat[:320].view(4, 5, 16)[:, :3], flat[40:360].view(4, 5, 16)[:, :3]
    assert not _apart(a, b)


@needs_lib
def test_binding_refuses_for_weigh_and_evict():
    import paper_2608_14648_amd as km
    torch, mode = _fake()
    with mode:
        dev = "cuda:0"

        def f(*shape, device=dev, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=device)

        def i(*shape, device=dev):
            return torch.empty(shape, dtype=torch.int32, device=device)

        cache = km.kv_cache(7, 2, 64, 16, torch.uint8, device=dev)
        seqs = km.KvSeqs(i(3, 4), i(3))
        q, lse, w = f(3, 4, 64, dtype=torch.bfloat16), f(3, 4), f(7, 2, 16)
        for a, err, msg in (((q, f(3, 2), w), ValueError, "lse must be"), ((q, f(4, 4), w), ValueError, "lse must be"),
                            ((q, lse.half(), w), TypeError, "lse"), ((q, f(3, 4, device="cuda:1"), w), ValueError, "lse must be on"),
                            ((q, lse, f(7, 2, 32)), ValueError, "weight must be"), ((q, lse, w.double()), TypeError, "weight"),
                            ((q, lse, f(7, 2, 16, device="cuda:1")), ValueError, "weight must be on"),
                            ((q, lse, f(7, 16, 2).transpose(1, 2)), ValueError, "contiguous"),
                            ((q[0], lse, w), ValueError, "q must be"), ((f(3, 4, 32), lse, w), ValueError, "q must be"),
                            ((q.float().requires_grad_(), lse, w), ValueError, "requires grad")):
            with pytest.raises(err, match=msg):
                km.kv_weigh(cache, seqs, *a)
        other = km.KvSeqs(i(3, 4, device="cuda:1"), i(3, device="cuda:1"))
        with pytest.raises(ValueError, match="sequences on"):
            km.kv_weigh(cache, other, q, lse, w)
        with pytest.raises(ValueError, match="sequences on"):
            km.kv_evict(cache, other, w, i(3), 5)
        for a, err, msg in (((w, i(2), 5), ValueError, "one number per sequence"), ((w, i(3).long(), 5), TypeError, "keep"),
                            ((w, i(3, device="cuda:1"), 5), ValueError, "keep must be on"), ((f(7, 2, 8), i(3), 5), ValueError, "weight")):
            with pytest.raises(err, match=msg):
                km.kv_evict(cache, seqs, *a)
        # numbers past 32 bits are the largest or -1, not their low halves
        from paper_2608_14648_amd import _kv
        seen = []

        class Lib:
            def kv_evict_bytes(self, cache, seqs, max_keep):
                seen.append(max_keep)
                return -1

            def km_last_error(self):
                return b"seen"

        for given, held in ((2 ** 32 + 5, 2 ** 31 - 1), (5, 5), (-2 ** 32 + 5, -1)):
            with pytest.MonkeyPatch.context() as m:
                m.setattr(_kv, "lib", Lib)
                with pytest.raises(km.KmqError, match="seen"):
                    km.kv_evict(cache, seqs, w, i(3), given)
            assert seen[-1] == held
