"""Scores that are infinite under a finite log-sum-exp: their key's weight is, and no other changes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,N,Nk", [(4, 2, 1, 300), (2, 2, 11, 100), (3, 1, 7, 900), (8, 1, 5, 66000), (4, 2, 70, 300), (5, 1, 33, 300), (2, 1, 127, 127), (10, 2, 13, 90)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("causal", [False, True])
def test_infinite_scores(H, Hkv, N, Nk, d, causal):
    import paper_2411_10958_amd as pa
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    print(f"infinite scores H={H}/{Hkv} N={N} Nk={Nk} d={d} causal={causal}", flush=True)
    q = torch.randn((1, H, N, d), generator=g, device="cuda").bfloat16()
    k = torch.randn((1, Hkv, Nk, d), generator=g, device="cuda").bfloat16()
    q[..., 1] = 1.0
    lse = torch.full((1, H, N), 5.0, device="cuda")
    lse[0, 0, 0] = math.inf if H > 1 else 5.0    # a query that gives every finite score a weight of zero
    clean = pa.sage_attn_key_weights(q, k, lse, causal=causal)
    assert clean.isfinite().all()
    key = Nk // 3 if not causal or Nk > N else Nk - 1                    # (one that the last query sees, and not the first one of head 0 alone)
    lse[0, 0, 0] = 5.0
    finite = pa.sage_attn_key_weights(q, k, lse, causal=causal)
    k[:, :, key, 1] = math.inf
    got = pa.sage_attn_key_weights(q, k, lse, causal=causal)
    torch.cuda.synchronize()
    others = torch.arange(Nk, device="cuda") != key
    assert (got[..., key] == math.inf).all() and torch.equal(got[..., others], finite[..., others])
    k[:, :, key, 1] = -math.inf
    got = pa.sage_attn_key_weights(q, k, lse, causal=causal)
    assert (got[..., key] == 0).all() and torch.equal(got[..., others], finite[..., others])
