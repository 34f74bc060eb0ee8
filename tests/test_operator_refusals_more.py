"""More of what the operators around attention refuse on the host, before anything is launched: no GPU."""

import pytest

from test_operator_refusals import EVICT, _pa, _status


@pytest.mark.parametrize("clear", [2, -1, 256])
def test_cache_evict_clear(clear):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_cache_evict", EVICT, clear=clear) == -2
