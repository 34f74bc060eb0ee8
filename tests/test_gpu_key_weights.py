"""The attention weight that keys have received, against float64."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _inputs(B, H, Hkv, N, Nk, d, dt, layout, causal=True, lens=None, sm_scale=0.0, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = ref.to_layout(torch.randn((B, H, N, d), generator=g, device="cuda").mul_(2.0).to(dt), layout)
    k = ref.to_layout(torch.randn((B, Hkv, Nk, d), generator=g, device="cuda").to(dt), layout)
    _, lse, _, _ = ref.shared_prefix(q, None, None, k, k, lens, causal, sm_scale, layout)
    return q, k, lse.float(), torch.rand((B, Hkv, Nk), generator=g, device="cuda").mul_(3.0)


def _check(pa, x, lens=None, causal=True, sm_scale=0.0, layout="HND", added=True):
    q, k, lse, w_in = x
    print(f"key weights q={tuple(q.shape)} k={tuple(k.shape)} {q.dtype} {layout} lens={None if lens is None else lens.tolist()} causal={causal} added={added}", flush=True)
    old = torch.full_like(w_in, 9.0)
    w = old.clone()
    got = pa.sage_attn_key_weights(q, k, lse, weights_in=w_in if added else None, weights=w, kv_lens=lens, causal=causal, sm_scale=sm_scale, layout=layout)
    torch.cuda.synchronize()
    assert got is w
    want, bound = ref.key_weights(q, k, lse, w_in if added else None, old, lens, causal, sm_scale, layout)
    ref.check("weights", got, want, bound)
    return got


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,Hkv,N,Nk", [(1, 1, 1, 1, 1), (2, 4, 2, 1, 300), (3, 8, 1, 5, 257), (2, 2, 2, 64, 64), (1, 6, 2, 65, 65), (2, 3, 3, 130, 520),
                                          (1, 4, 1, 700, 1000), (2, 8, 8, 200, 100)])
def test_sizes(B, H, Hkv, N, Nk, d):
    pa = _pa()
    dt, layout = (torch.bfloat16, "HND") if (B + N + d // 64) % 2 else (torch.float16, "NHD")
    for causal, added in ((True, True), (False, False)):
        _check(pa, _inputs(B, H, Hkv, N, Nk, d, dt, layout, causal), causal=causal, layout=layout, added=added)
    lens = torch.randint(0, Nk + 1, (B,), generator=torch.Generator().manual_seed(N)).to(torch.int32).cuda()
    _check(pa, _inputs(B, H, Hkv, N, Nk, d, dt, layout, True, lens, 0.05), lens=lens, sm_scale=0.05, layout=layout)


def test_a_prompt_in_several_pieces():
    """So many queries that a key tile's are divided over workgroups."""
    pa = _pa()
    x = _inputs(1, 4, 1, 3000, 3000, 64, torch.bfloat16, "HND")
    a = pa.binding.sage_attn_key_weights_args()
    a.B, a.H, a.H_kv, a.N, a.N_kv, a.d, a.causal, a.dtype = 1, 4, 1, 3000, 3000, 64, 1, 1
    assert pa.sage_attn_key_weights_workspace_bytes(a) > 0
    got = _check(pa, x)
    assert torch.equal(got, pa.sage_attn_key_weights(*x[:3], weights_in=x[3]))      # and the same bits again
    total = got.double() - x[3].double()
    assert abs(total.sum().item() / (4 * 3000) - 1) < 1e-5                           # every query gives away a weight of 1


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("G,N", [(4, 1), (3, 7), (5, 8), (8, 8)])
def test_steps_on_long_caches(G, N, d):
    """Few rows on so many keys that a wavefront walks over many tiles, and that more than 32 rows count as few too."""
    pa = _pa()
    lens = torch.tensor([33001, 16389, 17, 1], dtype=torch.int32, device="cuda")
    dt, layout = (torch.bfloat16, "NHD") if N % 2 else (torch.float16, "HND")
    for causal, added in ((True, True), (False, False)):
        _check(pa, _inputs(4, G, 1, N, 33001, d, dt, layout, causal, lens), lens=lens, causal=causal, layout=layout, added=added)


def test_more_workgroups_than_a_grid_is_wide():
    """64 heads of 140001 queries: over 4 million workgroups; some of the keys."""
    pa = _pa()
    H, N, d = 64, 140001, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, k = (torch.randn((1, H, N, d), generator=g, device="cuda").half() for _ in range(2))
    lse = torch.rand((1, H, N), generator=g, device="cuda") + 11.0
    got = pa.sage_attn_key_weights(q, k, lse, causal=False)
    at = torch.tensor([0, 1, 255, 256, 70000, 139775, 139776, 140000], device="cuda")
    for h in (0, 31, 63):
        x = (q[:, h:h + 1], k[:, h:h + 1, at], lse[:, h:h + 1])
        want, bound = ref.key_weights(*x, None, torch.zeros((1, 1, 8), device="cuda"), None, False, 0.0, "HND")
        ref.check(f"head {h}", got[:, h:h + 1, at], want, bound)


def test_rows_without_keys_and_lengths_out_of_range():
    pa = _pa()
    lens = torch.tensor([0, -3, 5000, 1], dtype=torch.int32, device="cuda")
    x = _inputs(4, 2, 1, 3, 90, 128, torch.bfloat16, "HND", True, lens)
    assert (x[2][:2] == -math.inf).all()
    got = _check(pa, x, lens=lens)
    assert (got[:2] == 9).all()
    # a query that saw nothing adds nothing, also where the call shows it keys
    x[2][2, 1, 1] = -math.inf
    _check(pa, x, lens=lens)


def test_masked_places_may_hold_anything():
    pa = _pa()
    for layout in ("HND", "NHD"):
        lens = torch.tensor([65, 100], dtype=torch.int32, device="cuda")
        q, k, lse, w_in = _inputs(2, 4, 2, 2, 190, 128, torch.bfloat16, layout, True, lens)
        want = _check(pa, (q, k, lse, w_in), lens=lens, layout=layout)
        for b in range(2):
            ref.heads_first(k, layout)[b, :, lens[b].item():] = math.nan
            w_in[b, :, lens[b].item():] = math.nan
        got = pa.sage_attn_key_weights(q, k, lse, weights_in=w_in, kv_lens=lens, layout=layout)
        for b in range(2):
            n = lens[b].item()
            assert torch.equal(got[b, :, :n], want[b, :, :n]) and (got[b, :, n:] == 0).all()
    # a key that a query does not see does not reach it
    q, k, lse, w_in = _inputs(1, 1, 1, 100, 100, 64, torch.bfloat16, "HND")
    k[0, 0, 99] = math.nan
    got = pa.sage_attn_key_weights(q, k, lse)
    assert got[0, 0, :99].isfinite().all() and got[0, 0, 99].isnan()


def test_in_place_another_stream_and_replays():
    pa = _pa()
    q, k, lse, w = _inputs(3, 8, 2, 300, 900, 128, torch.bfloat16, "HND")
    want = pa.sage_attn_key_weights(q, k, lse, weights_in=w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = pa.sage_attn_key_weights(q, k, lse, weights_in=w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    state, mirror = w.clone(), w.clone()
    lens = torch.tensor([900, 300, 512], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.sage_attn_key_weights(q, k, lse, weights_in=state, weights=state, kv_lens=lens)
    for step in range(3):
        lens.sub_(13)
        graph.replay()
        pa.sage_attn_key_weights(q, k, lse, weights_in=mirror, weights=mirror, kv_lens=lens)
        torch.cuda.synchronize()
        assert torch.equal(state, mirror), step


def test_weights_of_the_quantized_attention():
    """With the log-sum-exp of sage_attn_fwd_ex, whose scores are quantized: every query still gives away about 1 in all.  (A row's
    weights are off by the error of its log-sum-exp and of single scores; the 8-bit scores are within 0.1 of the exact ones here,
    checked against that log-sum-exp itself.)"""
    pa = _pa()
    q, k, exact, _ = _inputs(2, 4, 2, 500, 500, 128, torch.bfloat16, "HND")
    _, lse = pa.sage_attn_fwd_ex(q, k, k, causal=True, mode="int8_fp8", return_lse=True)
    off = (lse - exact).abs().max().item()
    got = pa.sage_attn_key_weights(q, k, lse).double()
    want, bound = ref.key_weights(q, k, lse, None, torch.zeros_like(got), None, True, 0.0, "HND")
    ref.check("weights", got, want, bound)
    assert off < 0.1 and abs(got.sum().item() / (2 * 4 * 500) - 1) <= math.expm1(off) + 1e-5
