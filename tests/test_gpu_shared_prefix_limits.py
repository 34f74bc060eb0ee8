"""Attention over a shared prefix at the ends of its range."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def test_the_most_rows():
    """2^24 queries of 256 channels, with partial results to merge: a block of 4096 over and over, so that every row is known."""
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    d, P, n, block = 256, 400, 1 << 24, 4096
    print(f"shared prefix of {P} keys, {n} queries of {d}", flush=True)
    few = torch.randn((1, 1, block, d), generator=g, device="cuda").bfloat16()
    kp, vp = (torch.randn((1, P, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = few.reshape(block, d).repeat(n // block, 1).view(1, 1, n, d)
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, return_lse=True)
    torch.cuda.synchronize()
    want, wl, ob, lb = ref.shared_prefix(few, kp, vp, None, None, None, True, 0.0, "HND")
    ref.check("lse", lse[:, :, :block], wl, lb)
    ref.check("out", out[:, :, :block], want, ob)
    lse, out = lse.view(-1, block), out.view(-1, block, d)
    assert torch.equal(lse, lse[:1].expand_as(lse))
    for i in range(0, len(out), 256):
        assert torch.equal(out[i:i + 256], out[:1].expand(256, -1, -1)), i
