"""Norms with a partial rotation: channels that are not turned have no part in each other's results, whatever they hold."""
import math

import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 24), (64, 32), (128, 2), (128, 64), (128, 100), (256, 128), (256, 250)])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_values_that_are_not_finite(d, rot, interleaved, value):
    pa = _pa()
    f = pa.sage_rope_frequencies(rot)
    g = torch.Generator(device="cuda")
    g.manual_seed(d + rot)
    q = torch.randn((2, 3, 9, d), generator=g, device="cuda").bfloat16()
    dy = torch.randn((2, 3, 9, d), generator=g, device="cuda").bfloat16()
    w = torch.randn(d, generator=g, device="cuda").add_(1.0)
    pos = torch.arange(5, 14, dtype=torch.int32, device="cuda")
    for c in {rot, d - 1, (rot + d) // 2}:
        rest = torch.arange(d, device="cuda") != c
        print(f"not finite d={d} rot={rot} interleaved={interleaved} channel={c} {value}", flush=True)
        # an infinite value makes its row's root infinite: the others are zeros, and it is infinity / infinity
        x = q.clone()
        x[1, 1, 4, c] = value
        y = pa.sage_qk_norm_rope(x, None, f, w, positions=pos, interleaved=interleaved)
        assert y[1, 1, 4, c].isnan()
        assert (y[1, 1, 4][rest] == 0).all() if value == math.inf else y[1, 1, 4].isnan().all()
        # a weight's reaches its channel
        v = w.clone()
        v[c] = value
        y, clean = pa.sage_qk_norm_rope(q, None, f, v, positions=pos, interleaved=interleaved), pa.sage_qk_norm_rope(q, None, f, w, positions=pos, interleaved=interleaved)
        assert not y[..., c].isfinite().any() and torch.equal(y[..., rest], clean[..., rest])
        # and a gradient's the weight's gradient of its channel, and its own row of dx
        dg = dy.clone()
        dg[1, 1, 4, c] = value
        got = pa.sage_qk_norm_rope_bwd(dg, q, None, None, f, w, positions=pos, interleaved=interleaved)
        clean = pa.sage_qk_norm_rope_bwd(dy, q, None, None, f, w, positions=pos, interleaved=interleaved)
        assert not got[2][c].isfinite() and torch.equal(got[2][rest], clean[2][rest])
        other = torch.ones((2, 3, 9), dtype=torch.bool, device="cuda")
        other[1, 1, 4] = False
        assert torch.equal(got[0][other], clean[0][other]) and not got[0][1, 1, 4].isfinite().any()
