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
