"""Attention over pages where scores are far from zero: the largest weight of a row is 1 however large its score, and no factor of a score overflows by itself."""
import math

import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu

FORMS = [(1, 4), (5, 4), (12, 4), (70, 2)]              # (N, G): 16, 32, 64 and 128 rows to a workgroup


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _one_channel(q, exponents, seed):
    """q [B, H, N, d] of zeros but for a channel of each row, which is a power of two of either sign; that channel and the sign."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, H, N, d = q.shape
    at = torch.randint(d, (B, H, N, 1), generator=g, device="cuda")
    sign = torch.randint(2, (B, H, N, 1), generator=g, device="cuda") * 2 - 1
    e = exponents[torch.randint(len(exponents), (B, H, N, 1), generator=g, device="cuda")]
    q.scatter_(3, at, (sign * torch.exp2(e.double())).to(q.dtype))
    return at[..., 0], sign[..., 0]


def _mean_of_the_largest(c, at, sign, lens, window, dt):
    """Every row's score is a power of two times a code in one channel.  With codes 2^-9 apart at least and scores of 2^12 for that step, the keys with the row's largest code share
    the weight evenly, and the others' weights vanish.  The weight of each may be off by a common factor (a score's rounding), so that it is rounded to the 16-bit type, half a
    step; then come the FP32 sums of as many terms and some sixteen factors of joins, and the output's rounding."""
    B, H, N = at.shape
    Hkv, d = c["k_cache"].shape[1], c["k_cache"].shape[3]
    out, bound = (torch.zeros((B, H, N, d), dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        n = int(lens[b])
        t, p = torch.arange(n, device="cuda"), max(n - N, 0) + torch.arange(N, device="cuda")[:, None]
        see = (t <= p) & (t > p - window) if window else t <= p
        for h in range(H):
            keys, _ = pref.values(c, "k", b, h // (H // Hkv), n)
            vals, _ = pref.values(c, "v", b, h // (H // Hkv), n)
            s = (keys.t().contiguous()[at[b, h]] * sign[b, h, :, None]).masked_fill(~see, -math.inf)
            w = (s == s.amax(1, keepdim=True)).double()
            ties = w.sum(1, keepdim=True)
            w /= ties
            out[b, h] = w @ vals
            mean = w @ vals.abs()
            bound[b, h] = ref.HALF[dt] * (out[b, h].abs() + mean) + (ties + 16) * ref.F32 * mean + ref.TINY[dt]
    return out, bound


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("N,G", FORMS)
def test_weights_of_far_scores(N, G, d, dt):
    """Rows side by side whose scores are from 2^12 to beyond 2^100, in blocks that all of them see and in others, with keys cut into chunks and not."""
    pa = _pa()
    for cap, window in ((256, 0), (256, 70), (8192, 0)):
        B = 2 if cap == 256 else 1
        c = pref.filled(B, 2, cap, 32, d, dt, seed=N + d)
        c["k_scale"].view(torch.uint8).fill_(127 + 30)
        lens = torch.tensor([cap, 131][:B], dtype=torch.int32, device="cuda")
        q = torch.zeros((B, 2 * G, N, d), dtype=dt, device="cuda")
        # a code is at least 2^-9: scores of (2 to the) exponent + 30 - 9 - 4 at least
        at, sign = _one_channel(q, torch.tensor([-5, -3, -1, 0, 1, 2, 4, 6, 9, 14] if dt == torch.float16 else [-5, -2, 0, 1, 3, 5, 10, 30, 60, 80], device="cuda"), d + N)
        print(f"far scores N={N} G={G} d={d} {dt} cap={cap} window={window}", flush=True)
        got = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window)
        torch.cuda.synchronize()
        ref.check("out", got, *_mean_of_the_largest(c, at, sign, lens, window, dt))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 256])
def test_a_single_key_has_all_the_weight(d, dt):
    """However large its score.  Its weight may be off by a score's rounding, which divides out but for its own rounding to the 16-bit type: half a step, half another for the output,
    and eight FP32 ones."""
    pa = _pa()
    c = pref.filled(3, 2, 64, 32, d, dt, seed=4)
    lens = torch.tensor([1, 1, 1], dtype=torch.int32, device="cuda")
    want = torch.stack([torch.stack([pref.values(c, "v", b, h // 4, 1)[0][0] for h in range(8)]) for b in range(3)])[:, :, None]
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    for e in range(0, 90, 3):
        c["k_scale"].view(torch.uint8).fill_(127 + e)
        q = torch.randn((3, 8, 1, d), generator=g, device="cuda").mul_(100.0).to(dt)
        got = pa.sage_attn_paged(q, **c, kv_lens=lens)
        ref.check(f"scale 2^{e}", got, want, (2 * ref.HALF[dt] + 8 * ref.F32) * want.abs() + ref.TINY[dt])
