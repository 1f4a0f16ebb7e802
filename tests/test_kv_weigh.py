"""kv_weigh without a GPU: sequences without rows in the oracle, in the C ABI's checks and in the binding."""
import ctypes as ct
import math
import os

import numpy as np
import pytest

import oracle.kv_ops as ops
from test_kv_ops import FAKE, _args, _cache4, _fake

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_14648_amd", "libkmq.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libkmq.so not built (run __graft_entry__.build())")


@pytest.fixture(scope="module")
def kmq():
    from paper_2608_14648_amd import _kmq
    return _kmq


def test_oracle_decays_a_sequence_without_rows():
    c = _cache4(pages=3)
    w = np.full((3, 1, 16), 4.0)
    q = np.zeros((1, 1, 32))
    # the second of three sequences has a row; the third's length does not fit
    table, lens, starts = np.array([[0], [1], [2]]), [5, 2, 17], [0, 0, 1, 1]
    for decay, old in ((0.5, 2.0), (1.0, 4.0), (0.0, 0.0)):
        out, *_ = ops.weigh(c, table, lens, starts, q, np.array([[math.log(2.0)]]), w, 1.0, decay=decay)
        np.testing.assert_allclose(out[0, 0], [old] * 5 + [4.0] * 11)
        np.testing.assert_allclose(out[1, 0, :3], [old + 0.5, 0.5, 4.0])
        np.testing.assert_array_equal(out[2], w[2])


@needs_lib
def test_a_call_without_rows_is_checked_like_others(kmq):
    L = kmq.lib()
    c = _args(kmq)[0]

    def call(seqs=(), q=None, hq=4, scale=0.1, type_=1, lse=None, weight=FAKE, decay=1.0):
        s = _args(kmq, seqs={**dict(rows=0, max_rows=0), **dict(seqs)})[1]
        return L.kv_weigh(ct.byref(c), ct.byref(s), q, hq, scale, 1, 0, type_, lse, weight, decay, None, 0, None)

    assert call() == 0  # nothing to age
    assert call(dict(starts=FAKE, max_rows=5)) == 0
    for kw, msg in ((dict(weight=None), "NULL"), (dict(seqs=dict(table=None)), "NULL"), (dict(seqs=dict(lens=None)), "NULL"),
                    (dict(seqs=dict(table_ld=0)), "share"), (dict(seqs=dict(table_ld=3)), "table_ld"), (dict(decay=-1.0), "decay"),
                    (dict(hq=3), "q_heads"), (dict(scale=0.0), "scale")):
        assert call(**kw) == -1 and msg in L.km_last_error().decode(), (kw, L.km_last_error())
    # with rows, queries and their log-sum-exp are wanted, and rows have to be what they say
    for kw, msg in ((dict(seqs=dict(rows=3, max_rows=1)), "NULL"), (dict(seqs=dict(rows=3, max_rows=1), lse=FAKE), "q is NULL"),
                    (dict(seqs=dict(rows=4, max_rows=1), lse=FAKE), "without starts")):
        assert call(**kw) == -1 and msg in L.km_last_error().decode(), (kw, L.km_last_error())
    s = _args(kmq, seqs=dict(rows=0, max_rows=0))[1]
    assert L.kv_weigh_bytes(ct.byref(c), ct.byref(s), 4, 1, 0, 1) == 0


@needs_lib
def test_binding_passes_a_call_without_rows_on():
    import paper_2608_14648_amd as km
    from paper_2608_14648_amd import _kv
    torch, mode = _fake()
    seen = []

    class Lib:
        def kv_weigh_bytes(self, *a):
            return 0

        def kv_weigh(self, *a):
            seen.append(a[10])
            return 0

    with mode, pytest.MonkeyPatch.context() as m:
        def t(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device="cuda:0")
        m.setattr(_kv, "lib", Lib)
        m.setattr(_kv, "_raw_stream", lambda i: 0)
        cache = km.kv_cache(7, 2, 64, 16, torch.uint8, device="cuda:0")
        seqs = km.KvSeqs(t(3, 4, dtype=torch.int32), t(3, dtype=torch.int32), rows=0)
        km.kv_weigh(cache, seqs, t(0, 4, 64), t(0, 4), t(7, 2, 16), decay=0.25)
    assert seen == [0.25]
