"""Attention of a batch over a shared prefix and its own keys, against float64."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _inputs(B, H, Hkv, N, P, Nk, d, dt, layout, seed=0, spread=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    q = ref.to_layout(r(B, H, N, d).mul_(spread).to(dt), layout)
    kp, vp = (ref.heads_first(r(Hkv, P, d).to(dt), layout).contiguous() if P else None for _ in range(2))
    k, v = (ref.to_layout(r(B, Hkv, Nk, d).to(dt), layout) if Nk else None for _ in range(2))
    return q, kp, vp, k, v


def _check(pa, x, lens=None, causal=True, sm_scale=0.0, layout="HND", **kw):
    q, kp, vp, k, v = x
    print(f"shared prefix q={tuple(q.shape)} kp={None if kp is None else tuple(kp.shape)} k={None if k is None else tuple(k.shape)} {q.dtype} {layout} "
          f"lens={None if lens is None else lens.tolist()} causal={causal}", flush=True)
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, causal=causal, sm_scale=sm_scale, layout=layout, return_lse=True, **kw)
    torch.cuda.synchronize()
    want, wl, ob, lb = ref.shared_prefix(q, kp, vp, k, v, lens, causal, sm_scale, layout)
    ref.check("lse", lse, wl, lb)
    ref.check("out", out, want, ob)
    return out, lse


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,Hkv,N,P,Nk", [(1, 1, 1, 1, 1, 1), (1, 2, 1, 1, 0, 64), (2, 2, 2, 1, 64, 0), (3, 8, 2, 1, 65, 63), (2, 4, 4, 5, 130, 65),
                                            (5, 8, 1, 3, 1000, 200), (2, 6, 2, 33, 257, 129), (3, 8, 1, 40, 333, 700), (2, 2, 2, 1, 900, 0), (3, 8, 2, 1, 0, 900),
                                            (2, 8, 1, 40, 100, 60)])
def test_sizes(B, H, Hkv, N, P, Nk, d):
    pa = _pa()
    dt, layout = (torch.bfloat16, "HND") if (B + N + d // 64) % 2 else (torch.float16, "NHD")
    x = _inputs(B, H, Hkv, N, P, Nk, d, dt, layout)
    _check(pa, x, layout=layout)
    if Nk > 1:
        lens = torch.randint(0, Nk + 1, (B,), generator=torch.Generator().manual_seed(N)).to(torch.int32)
        lens[0] = Nk
        _check(pa, x, lens=lens.cuda(), layout=layout)
        _check(pa, x, lens=lens.cuda(), causal=False, sm_scale=0.03, layout=layout)


@pytest.mark.parametrize("rows", [(8, 4), (9, 4), (16, 4), (17, 4), (32, 4), (33, 4), (64, 8)])
def test_rows_of_the_prefix_around_the_tiles(rows):
    """B G rows: one wavefront's 32, two, a workgroup's 128, several."""
    pa = _pa()
    B, G = rows
    _check(pa, _inputs(B, 2 * G, 2, 1, 777, 100, 128, torch.bfloat16, "HND", seed=B))


@pytest.mark.parametrize("Nk", [70, 990])
def test_no_keys_at_all_and_lengths_out_of_range(Nk):
    pa = _pa()
    x = _inputs(4, 4, 2, 3, 0, Nk, 64, torch.bfloat16, "HND")
    lens = torch.tensor([0, -5, 1000, 2], dtype=torch.int32, device="cuda")
    out, lse = _check(pa, x, lens=lens)
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all()


@pytest.mark.parametrize("P", [50, 1000])
def test_what_stands_behind_a_length_is_not_read(P):
    pa = _pa()
    for layout in ("HND", "NHD"):
        q, kp, vp, k, v = _inputs(3, 4, 2, 2, P, 190, 128, torch.bfloat16, layout)
        lens = torch.tensor([0, 65, 100], dtype=torch.int32, device="cuda")
        want = _check(pa, (q, kp, vp, k, v), lens=lens, layout=layout)
        for b in range(3):
            for x in (k, v):
                ref.heads_first(x, layout)[b, :, lens[b].item():] = math.nan
        got = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, layout=layout, return_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("P", [300, 1000])
def test_large_scores_and_values_that_are_not_numbers(P):
    pa = _pa()
    x = _inputs(2, 4, 2, 1, P, 100, 128, torch.bfloat16, "HND", spread=60.0)             # a few keys take it all
    _check(pa, x)
    q, kp, vp, k, v = _inputs(2, 4, 2, 1, P, 100, 128, torch.bfloat16, "HND")
    clean = pa.sage_attn_shared_prefix(q, kp, vp, k, v, return_lse=True)
    q[0, 1] = math.nan                       # one query: its row and no other
    k[1, 1, 7, 3] = math.nan                 # one key of one sequence: its group's rows
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, return_lse=True)
    bad = torch.zeros(2, 4, dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 2] = bad[1, 3] = True
    assert out[bad].isnan().all() and lse[bad].isnan().all()
    assert torch.equal(out[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])


@pytest.mark.parametrize("d,H,P,Nk", [(64, 4, 70, 100), (128, 8, 70, 33), (256, 2, 65, 10), (64, 4, 1001, 700), (128, 64, 1001, 300), (256, 8, 1001, 130)])
def test_infinite_values_of_the_last_keys(d, H, P, Nk):
    """Their channels become infinite, as their sum is, and no other changes."""
    pa = _pa()
    for layout in ("HND", "NHD"):
        q, kp, vp, k, v = _inputs(2, H, 2, 1, P, Nk, d, torch.bfloat16, layout, seed=P)
        lens = torch.tensor([Nk, Nk - 3], dtype=torch.int32, device="cuda")
        clean = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, layout=layout, return_lse=True)
        ref.heads_first(v, layout)[1, :, Nk - 4, 5] = math.inf
        ref.heads_first(vp, layout)[:, P - 1, 9] = -math.inf
        out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, layout=layout, return_lse=True)
        out, was = ref.heads_first(out, layout), ref.heads_first(clean[0], layout)
        assert torch.equal(lse, clean[1]) and (out[1, ..., 5] == math.inf).all() and (out[..., 9] == -math.inf).all()
        same = torch.ones(d, dtype=torch.bool, device="cuda")
        same[5] = same[9] = False
        assert torch.equal(out[..., same], was[..., same]) and torch.equal(out[0, ..., 5], was[0, ..., 5])


@pytest.mark.parametrize("P", [70, 1000])
@pytest.mark.parametrize("d,H,N,Nk", [(64, 4, 2, 100), (128, 2, 5, 130), (128, 8, 40, 200), (256, 4, 40, 90), (256, 2, 3, 64)])
def test_what_a_later_token_holds_does_not_reach_an_earlier_query(d, H, N, Nk, P):
    """Keys and values of the chunk's own tokens that are not finite: queries before them have what they had, to the bit."""
    pa = _pa()
    q, kp, vp, k, v = _inputs(2, H, 2, N, P, Nk, d, torch.float16 if d == 64 else torch.bfloat16, "HND", seed=d)
    lens = torch.tensor([Nk, Nk - 3], dtype=torch.int32, device="cuda")
    clean = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, return_lse=True)
    r = N // 2                                  # the token of query r of sequence 1: keys from there on are odd
    t = Nk - 3 - N + r
    v[1, 1, t, 5], v[1, 1, t + 1 if r + 1 < N else t, d - 1] = math.inf, math.nan
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, return_lse=True)
    heads = torch.zeros(2, H, dtype=torch.bool, device="cuda")
    heads[1, H // 2:] = True                    # those of KV head 1
    assert torch.equal(out[~heads], clean[0][~heads]) and torch.equal(lse, clean[1])
    assert torch.equal(out[1, H // 2:, :r], clean[0][1, H // 2:, :r])
    assert (out[1, H // 2:, r:, 5] == math.inf).all() and out[1, H // 2:, -1, d - 1].isnan().all()
    same = torch.ones(d, dtype=torch.bool, device="cuda")
    same[5] = same[d - 1] = False
    assert torch.equal(out[1, H // 2:, r:][..., same], clean[0][1, H // 2:, r:][..., same])
    k[1, 1, t] = math.nan
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, return_lse=True)
    assert torch.equal(out[1, H // 2:, :r], clean[0][1, H // 2:, :r]) and torch.equal(lse[1, H // 2:, :r], clean[1][1, H // 2:, :r])
    assert lse[1, H // 2:, r:].isnan().all() and out[1, H // 2:, r:].isnan().all()


def test_lse_merges_with_other_keys():
    """The prefix alone and the own keys alone, merged by their log-sum-exps, are the whole."""
    pa = _pa()
    q, kp, vp, k, v = _inputs(3, 4, 2, 1, 400, 90, 64, torch.float16, "HND")
    whole, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, return_lse=True)
    a, la = pa.sage_attn_shared_prefix(q, kp, vp, return_lse=True)
    b, lb = pa.sage_attn_shared_prefix(q, None, None, k, v, return_lse=True)
    both = torch.logaddexp(la, lb)
    assert torch.allclose(both, lse, rtol=0, atol=1e-5)      # (values up to 10: 2^-24 of them, some ten times)
    merged = a.float() * (la - both).exp()[..., None] + b.float() * (lb - both).exp()[..., None]
    # each part rounds its output (half a step) and its P (half a step of values up to max |v|), and so does the whole
    bound = ref.HALF[q.dtype] * 4 * torch.cat([vp.float().abs().flatten(), v.float().abs().flatten()]).max()
    assert (merged - whole.float()).abs().max() <= bound


def test_offsets_beyond_31_bits():
    """A cache of more than 2^31 values: the last sequence's last keys."""
    pa = _pa()
    B, Hkv, Nk, d = 2, 4, 1100000, 256
    k = torch.zeros((B, Hkv, Nk, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    k[1, 3, -300:] = torch.randn((300, d), generator=g, device="cuda").to(k.dtype)
    v[1, 3, -300:] = torch.randn((300, d), generator=g, device="cuda").to(k.dtype)
    k[1, 3, :-300, 0] = -300.0                               # the others get nothing
    q = torch.randn((B, Hkv, 1, d), generator=g, device="cuda").to(k.dtype)
    q[..., 0] = 20.0
    out, lse = pa.sage_attn_shared_prefix(q, None, None, k, v, return_lse=True)
    small = (q[1:, 3:], None, None, k[1:, 3:, -300:].contiguous(), v[1:, 3:, -300:].contiguous())
    want, wl, ob, lb = ref.shared_prefix(*small, None, True, 0.0, "HND")
    ref.check("out", out[1:, 3:], want, ob)
    ref.check("lse", lse[1:, 3:], wl, lb)


def test_another_stream_replays_and_the_same_bits_again():
    pa = _pa()
    x = _inputs(6, 8, 2, 1, 1500, 600, 128, torch.bfloat16, "HND")
    q, kp, vp, k, v = x
    lens = torch.tensor([600, 1, 0, 77, 300, 599], dtype=torch.int32, device="cuda")
    want = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, return_lse=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, return_lse=True, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out = torch.empty_like(q)
    graphs = []
    for _ in range(2):                       # two graphs that share a workspace, replayed in turn on one stream
        graph = torch.cuda.CUDAGraph()
        if not graphs:
            a = pa.binding._shared_prefix_args(q, kp, vp, k, v, lens, out, True, 0.0, "HND", None)
            ws = torch.empty(pa.sage_attn_shared_prefix_workspace_bytes(a), dtype=torch.uint8, device="cuda")
        with torch.cuda.graph(graph):
            _, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, out=out, return_lse=True, workspace=ws)
        graphs.append((graph, lse))
    for step in range(4):
        graph, lse = graphs[step % 2]
        lens.copy_((lens + 31 * step) % 601)
        q.mul_(-1.0)
        ws.fill_(255)                        # nothing is kept from call to call
        graph.replay()
        again = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, return_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1]), step
