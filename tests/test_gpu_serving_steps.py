"""The operators together, as a serving program uses them: a prompt that all sequences share, a few tokens of each sequence's own, and a
cache that is cut back to its bound by the weight its keys have received."""
import torch

import pytest

import operator_reference as ref

pytestmark = pytest.mark.gpu


def test_generation_over_a_shared_prompt_with_a_bounded_cache():
    import paper_2411_10958_amd as pa
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    B, H, Hkv, d, P, cap, bound_to, recent = 4, 8, 2, 128, 400, 12, 8, 3
    dt = torch.bfloat16
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)
    f = pa.sage_rope_frequencies(d, base=500000.0)
    # the prompt: rotated, attended to by the quantized path, its cache kept
    qp, kp0, vp = r(1, H, P, d), r(1, Hkv, P, d), r(1, Hkv, P, d)
    qp, kp = pa.sage_rope(qp, kp0, f)
    ref.check("prompt keys", kp, *ref.rope(kp0, f, torch.arange(P, device="cuda"), False, False, 1.0, "HND"))
    out = pa.sage_attn_fwd_ex(qp, kp, vp, causal=True)
    assert out.isfinite().all()
    k = torch.zeros((B, Hkv, cap, d), dtype=dt, device="cuda")
    v, w = torch.zeros_like(k), torch.zeros((B, Hkv, cap), device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    evictions = 0
    for step in range(20):
        pos = torch.full((B, 1), P + step, dtype=torch.int32, device="cuda")
        n = int(lens[0])
        q = r(B, H, 1, d)
        pa.sage_rope(q, r(B, Hkv, 1, d), f, positions=pos, q_out=q, k_out=k[:, :, n:n + 1])       # straight into the cache
        v[:, :, n] = r(B, Hkv, d)
        w[:, :, n] = 0
        lens += 1
        o, lse = pa.sage_attn_shared_prefix(q, kp[0], vp[0], k, v, kv_lens=lens, return_lse=True)
        want, wl, ob, lb = ref.shared_prefix(q, kp[0], vp[0], k, v, lens, True, 0.0, "HND")
        ref.check(f"output of step {step}", o, want, ob)
        ref.check(f"lse of step {step}", lse, wl, lb)
        ww, wb = ref.key_weights(q, k, lse, w, w, lens, True, 0.0, "HND")
        pa.sage_attn_key_weights(q, k, lse, weights_in=w, weights=w, kv_lens=lens)
        ref.check(f"weights of step {step}", w, ww, wb.clamp(min=1e-30))
        if int(lens[0]) == cap:
            keep = ref.evict(k, v, w, bound_to, 0, recent, lens, "HND")
            ko, vo, wo, kept, left = pa.sage_cache_evict(k, v, w, bound_to, recent=recent, kv_lens=lens)
            assert kept.tolist() == keep and left.tolist() == [bound_to] * B
            k[:, :, :bound_to], v[:, :, :bound_to], w[:, :, :bound_to] = ko, vo, wo
            lens.copy_(left)
            evictions += 1
    # 12 tokens, then 4 more each time: cut back at steps 12, 16 and 20
    assert evictions == 3 and int(lens[0]) == bound_to
