"""Attention over pages with scores of minus infinity: weights of zero beside finite ones; a row that has no others is not a row that sees nothing."""
import math

import pytest
import torch

import operator_reference as ref
import paged_reference as pref
from test_gpu_paged_far_scores import FORMS, _pa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,G", FORMS)
def test_scores_of_minus_infinity(N, G, dt):
    pa = _pa()
    for d, cap, window in ((64, 256, 0), (64, 8192, 0), (128, 256, 70), (256, 256, 0), (256, 8192, 70)):
        B = 2 if cap == 256 else 1
        c = pref.filled(B, 2, cap, 32, d, dt, seed=N)
        lens = torch.tensor([cap - 3, 131][:B], dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda")
        g.manual_seed(N + d)
        q = torch.randn((B, 2 * G, N, d), generator=g, device="cuda").to(dt)
        print(f"minus infinity N={N} G={G} d={d} {dt} cap={cap} window={window}", flush=True)
        c["k_cache"].view(torch.uint8)[..., 7] = 0x08          # a channel of small positive codes
        clean = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window, return_lse=True)
        hit = torch.zeros((B, 2 * G, N), dtype=torch.bool, device="cuda")
        hit[0, 1, N // 2] = hit[0, G, N - 1] = True
        bad = q.clone()
        bad[..., 7] = torch.where(hit, -math.inf, bad[..., 7])
        got = pa.sage_attn_paged(bad, **c, kv_lens=lens, window=window, return_lse=True)
        torch.cuda.synchronize()
        assert got[0][hit].isnan().all() and (got[1][hit].isnan() | (got[1][hit] == -math.inf)).all()
        assert torch.equal(got[0][~hit], clean[0][~hit]) and torch.equal(got[1][~hit], clean[1][~hit])
        none = pa.sage_attn_paged(bad, **c, kv_lens=torch.zeros_like(lens), window=window, return_lse=True)      # (no token: zeros, whatever the query is)
        assert (none[0] == 0).all() and (none[1] == -math.inf).all()


@pytest.mark.parametrize("N,G", FORMS)
def test_minus_infinity_beside_finite_scores(N, G):
    """Scores beyond FP32's range downwards have no weight beside one in it, wherever in the cache either is."""
    pa = _pa()
    for d, cap in ((64, 256), (128, 8192), (256, 8192)):
        c = pref.filled(1, 2, cap, 32, d, torch.bfloat16, seed=N)
        c["k_scale"].view(torch.uint8).fill_(127 + 60)
        q = torch.zeros((1, 2 * G, N, d), dtype=torch.bfloat16, device="cuda")
        q[..., 3] = -2.0 ** 90
        for seen in ([0], [5, 100], [cap - N - 1, 33]):
            codes = c["k_cache"].view(torch.uint8)
            codes[..., 3] = 0x38                                # 1
            for t in seen:
                codes[int(c["page_table"][0, t // 32]), :, t % 32, 3] = 0
            got, lse = pa.sage_attn_paged(q, **c, return_lse=True)
            want = torch.stack([pref.values(c, "v", 0, h // G, cap)[0][seen] for h in range(2 * G)])[None, :, None]      # [1, H, 1, seen, d]
            mean, size = want.mean(3), want.abs().mean(3)
            ref.check("out", got, mean.expand(1, 2 * G, N, d), ((2.0 ** -8 + 2.0 ** -20) * size + 2.0 ** -8 * mean.abs() + 2.0 ** -134).expand(1, 2 * G, N, d))
            assert ((lse - math.log(len(seen))).abs() <= 2.0 ** -20).all()
