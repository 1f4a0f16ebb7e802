"""What the binding of the key/value cache takes and refuses beyond test_kv.py and test_kv_ops.py; without a GPU."""
import os

import pytest

from test_kv_ops import _fake

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_14648_amd", "libkmq.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libkmq.so not built (run __graft_entry__.build())")


@needs_lib
def test_strides_of_no_rows_mean_nothing():
    import paper_2608_14648_amd as km
    torch, mode = _fake()
    with mode:
        def t(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device="cuda:0")
        cache = km.kv_cache(7, 2, 64, 16, device="cuda:0")
        seqs = km.KvSeqs(t(3, 4, dtype=torch.int32), t(3, dtype=torch.int32), rows=0)
        odd = torch.empty_strided((0, 2, 64), (1, 1, 2), dtype=torch.bfloat16, device="cuda:0")
        km.kv_write(cache, seqs, odd, odd)
        km.kv_read(cache, seqs, torch.bfloat16, k=odd, v=t(0, 2, 64))
        out, _ = km.kv_attend(cache, seqs, odd)
        assert tuple(out.shape) == (0, 2, 64)
        rot = km.KvRotary(t(8, dtype=torch.float64))
        assert tuple(km.kv_rotate(rot, seqs, odd, odd)[1].shape) == (0, 2, 64)
        # of some rows they do
        one = km.KvSeqs(t(3, 4, dtype=torch.int32), t(3, dtype=torch.int32))
        with pytest.raises(ValueError, match="contiguous"):
            km.kv_attend(cache, one, torch.empty_strided((3, 2, 64), (256, 128, 2), dtype=torch.bfloat16, device="cuda:0"))


@needs_lib
def test_rows_turned_in_place_are_not_read_for_others():
    """q_out may be q's own rows, but then k must not be read from them: neither as the same tensor nor as a view, and the other way round."""
    import paper_2608_14648_amd as km
    torch = pytest.importorskip("torch")
    from paper_2608_14648_amd._kv import _check_outputs
    buf = torch.empty((6, 10, 16))
    x, y, z = buf[:, :3], buf[:, 3:6], buf[:, 6:9]
    view = buf[:, :3]
    # in place, apart, or not given
    for q, k, q_out, k_out in ((x, y, x, y), (x, y, view, y), (x, None, x, None), (x, y, x, z), (x, y, z, y), (x, x, y, z), (x, x, y, None),
                               (x, y, None, y)):
        _check_outputs(q, k, q_out, k_out)
    for q, k, q_out, k_out in ((x, x, x, None), (x, x, x, y), (x, x, None, x), (x, x, y, x), (x, view, x, y), (view, x, x, y),
                               (x, view, y, x), (x, x, view, None), (x, x, x, x), (x, y, y, None), (x, y, None, x), (x, y, y, x)):
        with pytest.raises(ValueError, match="overlap"):
            _check_outputs(q, k, q_out, k_out)


@needs_lib
def test_in_place_whatever_the_stride_of_an_axis_of_one():
    import paper_2608_14648_amd as km  # noqa: F401
    torch = pytest.importorskip("torch")
    from paper_2608_14648_amd._kv import _check_outputs
    buf = torch.empty(1000)
    for shape, a, b in (((1, 3, 16), (160, 16, 1), (48, 16, 1)), ((5, 1, 16), (160, 16, 1), (160, 160, 1)), ((1, 1, 16), (1, 1, 1), (16, 16, 1))):
        _check_outputs(buf.as_strided(shape, a), None, buf.as_strided(shape, b), None)
    for shape, a, b in (((2, 3, 16), (160, 16, 1), (48, 16, 1)), ((5, 2, 16), (160, 16, 1), (160, 80, 1))):
        with pytest.raises(ValueError, match="same rows"):
            _check_outputs(buf.as_strided(shape, a), None, buf.as_strided(shape, b), None)
