"""Rope on tensors that lie between each other without sharing a value: allowed, and right."""
import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def test_tensors_that_interleave():
    import paper_2411_10958_amd as pa
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    B, H, Hkv, N, d = 2, 4, 2, 33, 64
    f = pa.sage_rope_frequencies(d)
    pos = torch.arange(N, device="cuda")
    buf = torch.randn((B, N, 2 * (H + Hkv), d), generator=g, device="cuda").bfloat16()
    old = buf.clone()
    q, k, qo, ko = buf[:, :, :H], buf[:, :, H:H + Hkv], buf[:, :, H + Hkv:2 * H + Hkv], buf[:, :, 2 * H + Hkv:]
    # outputs beside the inputs, in the same buffer
    pa.sage_rope(q, k, f, layout="NHD", q_out=qo, k_out=ko)
    ref.check("q", qo, *ref.rope(old[:, :, :H], f, pos, False, False, 1.0, "NHD"))
    ref.check("k", ko, *ref.rope(old[:, :, H:H + Hkv], f, pos, False, False, 1.0, "NHD"))
    assert torch.equal(buf[:, :, :H + Hkv], old[:, :, :H + Hkv])
    # q in place, k into the other tokens of its own rows' heads
    buf.copy_(old)
    even, odd = buf[:, 0:32:2, H:H + Hkv], buf[:, 1:33:2, H:H + Hkv]
    pa.sage_rope(buf[:, 0:32:2, :H], even, f, layout="NHD", q_out=buf[:, 0:32:2, :H], k_out=odd)
    ref.check("k", odd, *ref.rope(old[:, 0:32:2, H:H + Hkv], f, pos[:16], False, False, 1.0, "NHD"))
    ref.check("q", buf[:, 0:32:2, :H], *ref.rope(old[:, 0:32:2, :H], f, pos[:16], False, False, 1.0, "NHD"))
    assert torch.equal(buf[:, 1::2, :H], old[:, 1::2, :H]) and torch.equal(even, old[:, 0:32:2, H:H + Hkv])
    # a token later: some rows would be read after they are written
    for kw in (dict(q_out=buf[:, 1:, :H]), dict(q_out=buf[:, :-1, 1:H + 1])):
        with pytest.raises(pa.SageError):
            pa.sage_rope(buf[:, :-1, :H], None, f, layout="NHD", **kw)
