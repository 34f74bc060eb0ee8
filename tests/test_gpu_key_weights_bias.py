"""Key weights at large log-sum-exps: what is off is a rounding of each query's own, not a share that all have in common."""
import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 65])               # (few rows, and tiles of queries: 64 of the 65 have lse = +inf and add zeros)
@pytest.mark.parametrize("d,sm_scale", [(64, 0.0), (128, 0.0), (256, 0.0), (128, 0.05)])
def test_errors_of_the_exponents_average_out(d, sm_scale, N):
    """4096 queries with a head each, scores around 80 from one channel (their products are exact).  The mean relative error of all
    weights: the constant -lse log2 e, around 118, is rounded by 2^-18 at most, 2^-18 / sqrt(3) in the middle, times ln 2, and over 4096 of them
    six times 1 / sqrt(4096) of that; scale log2 e by 2^-24 of a difference of 3; the exponential by 2^-23."""
    import paper_2411_10958_amd as pa
    g = torch.Generator(device="cuda")
    g.manual_seed(d + N)
    B, H, Nk = 64, 64, 64
    scale = sm_scale or 1 / math.sqrt(d)
    print(f"bias d={d} sm_scale={sm_scale} N={N}", flush=True)
    q, k = torch.zeros((B, H, N, d), device="cuda", dtype=torch.bfloat16), torch.zeros((B, H, Nk, d), device="cuda", dtype=torch.bfloat16)
    q[..., 5] = 32.0
    k[..., 5] = (80 + 2 * (torch.rand((B, H, Nk), generator=g, device="cuda") - 0.5)) / (32 * scale)
    lse = torch.full((B, H, N), math.inf, device="cuda")
    lse[..., N // 2] = 81 + torch.rand((B, H), generator=g, device="cuda")
    got = pa.sage_attn_key_weights(q, k, lse, causal=False, sm_scale=sm_scale)
    scale = ctypes.c_float(sm_scale).value or scale                       # (the argument is an FP32 number: 0.05 is 1.5e-8 of itself more there)
    want = torch.exp(32.0 * k[..., 5].double() * scale - lse[..., N // 2, None].double())
    off = (got.double() / want - 1).mean().item()
    bound = 6 * 2.0 ** -18 / math.sqrt(3) * math.log(2) / math.sqrt(4096) + 3 * 2.0 ** -24 + 2.0 ** -23
    assert abs(off) <= bound, (off, bound)
