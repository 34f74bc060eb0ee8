"""Attention over pages refuses an sm_scale that is no factor in FP32: no GPU."""
import pytest

from test_paged_refusals import PAGED, _pa, _status


@pytest.mark.parametrize("sm_scale", [2.4e38, 3.4e38])
def test_scale_beyond_fp32(sm_scale):
    """Scores are to the base 2: times log2(e) it has to be finite."""
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_paged", PAGED, sm_scale=sm_scale) == -1
    assert _status(pa, lib, "sage_attn_paged", PAGED, sm_scale=2.3e38, workspace=0, max_pages=4096) == -3      # (this far, and the workspace is asked for)
