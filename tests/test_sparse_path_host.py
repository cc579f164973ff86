"""What SparseAttention refuses when it is made: sizes that none of its calls would take."""
import pytest

from paper_2608_17995_amd.step import SparseAttention

OK = dict(rows=128, H=2, d=64, keep=1, dims=(64,))


@pytest.mark.parametrize("bad", [dict(batch=17), dict(batch=1 << 40), dict(H=1025), dict(H=2048, Hk=2), dict(keep=-1), dict(lead=-1),
                                 dict(Hk=-2), dict(Hk=0), dict(Hk=4), dict(H=0), dict(d=32), dict(rows=0), dict(rows=(1 << 31) - 4096),
                                 dict(dims=(16, 56))])
def test_refused(bad):
    with pytest.raises(ValueError, match="SparseAttention: rows"):
        SparseAttention(**{**OK, **bad})
