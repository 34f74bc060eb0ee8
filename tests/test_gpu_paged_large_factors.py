"""Attention over pages where sm_scale times a block's scale is beyond FP32, and the scores are not."""
import pytest
import torch

import operator_reference as ref
import paged_reference as pref
from test_gpu_paged_far_scores import FORMS, _mean_of_the_largest, _one_channel, _pa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N,G", FORMS)
def test_scores_of_zero(N, G, dt):
    """Queries of zeros give every token they see the same weight."""
    pa = _pa()
    for d in (64, 128, 256):
        for byte, sm_scale in ((127 + 119, 1000.0), (254, 2.0), (254, 1e38)):
            c = pref.filled(2, 2, 256, 32, d, dt, seed=N)
            q = torch.zeros((2, 2 * G, N, d), dtype=dt, device="cuda")
            lens = torch.tensor([256, 131], dtype=torch.int32, device="cuda")
            want, _, bound, _ = pref.paged(q, c, lens, None, True, 0, 0, sm_scale, "HND")
            c["k_scale"].view(torch.uint8).fill_(byte)
            print(f"zero scores N={N} G={G} d={d} {dt} scale byte {byte} sm_scale {sm_scale}", flush=True)
            got = pa.sage_attn_paged(q, **c, kv_lens=lens, sm_scale=sm_scale)
            torch.cuda.synchronize()
            ref.check("out", got, want, bound)


@pytest.mark.parametrize("N,G", FORMS)
def test_scores_of_tiny_queries(N, G):
    """bf16 queries so small that scores are ordinary again: 2^-112 and less times codes of 2^119."""
    pa = _pa()
    for d in (64, 128, 256):
        for window in (0, 70):
            c = pref.filled(2, 2, 256, 32, d, torch.bfloat16, seed=N)
            c["k_scale"].view(torch.uint8).fill_(127 + 119)
            q = torch.zeros((2, 2 * G, N, d), dtype=torch.bfloat16, device="cuda")
            lens = torch.tensor([256, 131], dtype=torch.int32, device="cuda")
            at, sign = _one_channel(q, torch.tensor([-112, -110, -106], device="cuda"), N)
            got = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window, sm_scale=2.0 ** 14)
            torch.cuda.synchronize()
            ref.check("out", got, *_mean_of_the_largest(c, at, sign, lens, window, torch.bfloat16))
