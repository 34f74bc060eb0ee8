"""Whole numbers that do not fit their field are refused by the operators around attention; they do not come back as others."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_numbers_that_do_not_fit():
    import paper_2411_10958_amd as pa
    x = torch.zeros((1, 2, 90, 64), device="cuda", dtype=torch.bfloat16)
    w = torch.zeros((1, 2, 90), device="cuda")
    f = pa.sage_rope_frequencies(64)
    for offset in (1 << 64, (1 << 64) + 5, -(1 << 64), 1 << 63, 1 << 53):
        with pytest.raises(pa.SageError):
            pa.sage_rope(x, None, f, offset=offset)
    for kw in (dict(sink=1 << 32), dict(recent=(1 << 32) + 7), dict(sink=-(1 << 32)), dict(recent=1 << 31), dict(sink=-1)):
        with pytest.raises(pa.SageError):
            pa.sage_cache_evict(x, x, w, 30, **kw)
    assert pa.sage_rope(x, None, f, offset=1 << 52) is not None
