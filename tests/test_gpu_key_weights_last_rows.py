"""Key weights where the last tile of queries is not full: the places behind the last query repeat it, and must not count."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _inputs(B, H, Hkv, N, Nk, d, dt, layout, causal, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = ref.to_layout(torch.randn((B, H, N, d), generator=g, device="cuda").to(dt), layout)
    k = ref.to_layout(torch.randn((B, Hkv, Nk, d), generator=g, device="cuda").to(dt), layout)
    _, lse, _, _ = ref.shared_prefix(q, None, None, k, k, None, causal, 0.0, layout)
    return q, k, lse.float()


# (per head with a last tile of 6 and of 63 rows; a group's rows in one list: 165, 65, 127; few rows)
@pytest.mark.parametrize("H,Hkv,N,Nk", [(4, 2, 70, 300), (2, 1, 127, 127), (5, 1, 33, 300), (10, 2, 13, 90), (2, 2, 1, 100), (6, 1, 3, 700), (5, 1, 13, 20)])
@pytest.mark.parametrize("d,dt,layout", [(64, torch.float16, "NHD"), (128, torch.bfloat16, "HND"), (256, torch.bfloat16, "NHD")])
@pytest.mark.parametrize("causal", [False, True])
def test_a_last_query_that_saw_nothing_adds_nothing_whatever_it_holds(H, Hkv, N, Nk, d, dt, layout, causal):
    """lse = -inf: places of a padded chunk that nobody wrote.  The same bits as with finite queries there, and the formula's values."""
    pa = _pa()
    q, k, lse = _inputs(2, H, Hkv, N, Nk, d, dt, layout, causal)
    print(f"last queries H={H}/{Hkv} N={N} Nk={Nk} d={d} {dt} {layout} causal={causal}", flush=True)
    lse[0, :, -1] = -math.inf                    # of every head of one sequence, of the last head of the other
    lse[1, -1, -1] = -math.inf
    old = torch.zeros((2, Hkv, Nk), device="cuda")
    want, bound = ref.key_weights(q, k, lse, None, old, None, causal, 0.0, layout)
    clean = pa.sage_attn_key_weights(q, k, lse, causal=causal, layout=layout)
    ref.check("finite", clean, want, bound)
    for odd in (math.nan, math.inf, -math.inf):
        heads = ref.heads_first(q, layout)
        heads[0, :, -1], heads[1, -1, -1] = odd, odd
        got = pa.sage_attn_key_weights(q, k, lse, causal=causal, layout=layout)
        torch.cuda.synchronize()
        assert torch.equal(got, clean), odd
