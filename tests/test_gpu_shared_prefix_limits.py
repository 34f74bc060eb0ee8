"""Attention over a shared prefix at the ends of its range."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def test_the_most_rows():
    """2^24 queries of 256 channels, with partial results to merge: a block of 4096 over and over, so that every row is known."""
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    d, P, n, block = 256, 400, 1 << 24, 4096
    print(f"shared prefix of {P} keys, {n} queries of {d}", flush=True)
    few = torch.randn((1, 1, block, d), generator=g, device="cuda").bfloat16()
    kp, vp = (torch.randn((1, P, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = few.reshape(block, d).repeat(n // block, 1).view(1, 1, n, d)
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, return_lse=True)
    torch.cuda.synchronize()
    want, wl, ob, lb = ref.shared_prefix(few, kp, vp, None, None, None, True, 0.0, "HND")
    ref.check("lse", lse[:, :, :block], wl, lb)
    ref.check("out", out[:, :, :block], want, ob)
    lse, out = lse.view(-1, block), out.view(-1, block, d)
    assert torch.equal(lse, lse[:1].expand_as(lse))
    for i in range(0, len(out), 256):
        assert torch.equal(out[i:i + 256], out[:1].expand(256, -1, -1)), i


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,H,N,P,Nk", [(64, 2, 1, 500, 200), (128, 2, 1, 300, 100), (256, 2, 1, 100, 100), (64, 8, 1, 20000, 3000), (128, 8, 40, 9000, 700), (256, 4, 5, 9000, 700)])
def test_weights_far_below_the_largest(d, H, N, P, Nk, dt):
    """Every 64th key gets e^18.5 times the weight of the others, and has values of zero: the output is what the others add up to,
    each 2^-26.7 of the largest.  All of them are positive, so the output is off by half a step for P and half a step for itself; scores of 18.5
    are exact, and with the constant log2 e and the exponent's two roundings at 26.7 a weight is off by less than 2^-18."""
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(P)
    print(f"small weights d={d} H={H} N={N} P={P} Nk={Nk} {dt}", flush=True)
    q = torch.zeros((2, H, N, d), device="cuda", dtype=dt)
    q[..., 3] = 1.0
    def cache(*shape):
        k = torch.zeros((*shape, d), device="cuda", dtype=dt)
        v = (torch.rand((*shape, d), generator=g, device="cuda") * 1000 + 500).to(dt)
        k[..., ::64, 3], v[..., ::64, :] = 18.5, 0.0
        return k, v
    kp, vp = cache(2, P)
    k, v = cache(2, 2, Nk)
    lens = torch.tensor([Nk, Nk - 7], dtype=torch.int32, device="cuda")
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=lens, sm_scale=1.0, return_lse=True)
    want, wl, _, lb = ref.shared_prefix(q, kp, vp, k, v, lens, True, 1.0, "HND")
    ref.check("lse", lse, wl, lb)
    assert want.min() > 1e-4
    ref.check("out", out, want, ref.TINY[dt] + (2.01 * ref.HALF[dt] + 2.0 ** -18) * want.abs())


def test_scores_beyond_all_reason():
    """Of a size at which FP32 has no halves any more (fp16): the largest takes all, as in the formula.  (P and the output are off by half a
    step each; the log-sum-exp by four FP32 roundings of its size.)"""
    pa = _pa()
    d = 128
    for size in (2.0 ** 10, 2.0 ** 12, 2.0 ** 13):                       # scores of sign times size^2 = 2^20, 2^24, 2^26, in units of log 2 1.44 times that
        q = torch.zeros((1, 2, 1, d), device="cuda", dtype=torch.float16)
        q[0, 0, 0, 0], q[0, 1, 0, 0] = size, -size
        kp = torch.zeros((2, 1000, d), device="cuda", dtype=torch.float16)
        kp[:, :, 0] = size / 2
        kp[:, 5, 0], kp[:, 900, 0] = size, -size
        vp = torch.rand((2, 1000, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
        out, lse = pa.sage_attn_shared_prefix(q, kp, vp, sm_scale=1.0, return_lse=True)
        want = torch.stack([vp[0, 5], vp[1, 900]])[None, :, None].double()
        ref.check(f"out of {size}", out, want, ref.TINY[torch.float16] + (2 * ref.HALF[torch.float16] + 2.0 ** -20) * want)
        assert (lse - size * size).abs().max() <= 2.0 ** -22 * size * size


@pytest.mark.parametrize("B,H,N,P,Nk,d", [(2, 4, 1, 70, 60, 128), (2, 8, 40, 100, 60, 64), (3, 8, 5, 1000, 300, 128), (2, 8, 70, 500, 300, 256)])
@pytest.mark.parametrize("layout", ["HND", "NHD"])
def test_the_output_in_place_of_the_queries(B, H, N, P, Nk, d, layout):
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(P)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    q, k, v = (ref.to_layout(r(B, h, n, d), layout) for h, n in ((H, N), (2, Nk), (2, Nk)))
    kp, vp = (ref.heads_first(r(2, P, d), layout).contiguous() for _ in range(2))
    want, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, layout=layout, return_lse=True)
    got, lse2 = pa.sage_attn_shared_prefix(q, kp, vp, k, v, layout=layout, return_lse=True, out=q)
    assert got is q and torch.equal(got, want) and torch.equal(lse2, lse)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,N,P,Nk", [(1, 8, 1, 131072, 512), (1, 4, 3, 0, 140001), (2, 2, 1, 140001, 0), (1, 2, 5, 90000, 60001)])
def test_one_head_of_many_keys(B, H, N, P, Nk, d):
    """As many partial results to merge as there can be."""
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    print(f"one head B={B} H={H} N={N} P={P} Nk={Nk} d={d}", flush=True)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    q = r(B, H, N, d)
    kp, vp = (r(1, P, d) if P else None for _ in range(2))
    k, v = (r(B, 1, Nk, d) if Nk else None for _ in range(2))
    out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, return_lse=True)
    want, wl, ob, lb = ref.shared_prefix(q, kp, vp, k, v, None, True, 0.0, "HND")
    ref.check("lse", lse, wl, lb)
    ref.check("out", out, want, ob)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_caches_without_any_place(d):
    """No prefix and no own keys: zeros and -inf; and each of them empty beside the other."""
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    for H, N in ((4, 1), (2, 300)):
        q, none, own = r(3, H, N, d), r(2, 0, d), r(3, 2, 0, d)
        lens = torch.tensor([0, 5, -1], dtype=torch.int32, device="cuda")
        for args in ((none, none, own, own), (none, none), (None, None, own, own)):
            out, lse = pa.sage_attn_shared_prefix(q, *args, kv_lens=lens if len(args) > 2 else None, out=torch.full_like(q, 3.0), return_lse=True)
            assert (out == 0).all() and (lse == -math.inf).all()
        kp, vp, k, v = r(2, 700, d), r(2, 700, d), r(3, 2, 400, d), r(3, 2, 400, d)
        for a, b in (((kp, vp, own, own), (kp, vp)), ((none, none, k, v), (None, None, k, v))):
            x, y = (pa.sage_attn_shared_prefix(q, *args, return_lse=True) for args in (a, b))
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


@pytest.mark.parametrize("B,H,N,P,Nk", [(1, 4, 513, 700, 600), (2, 2, 1000, 300, 1300), (3, 4, 130, 200, 60), (1, 8, 257, 0, 300)])
@pytest.mark.parametrize("d,dt,layout", [(64, torch.float16, "NHD"), (128, torch.bfloat16, "HND"), (256, torch.bfloat16, "NHD")])
def test_chunks_of_a_prompt(B, H, N, P, Nk, d, dt, layout):
    """Many queries over a prefix and their own keys, also with fewer keys than queries."""
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    print(f"chunk B={B} H={H} N={N} P={P} Nk={Nk} d={d} {dt} {layout}", flush=True)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)
    q, k, v = ref.to_layout(r(B, H, N, d), layout), ref.to_layout(r(B, 2, Nk, d), layout), ref.to_layout(r(B, 2, Nk, d), layout)
    kp, vp = (ref.heads_first(r(2, P, d), layout).contiguous() if P else None for _ in range(2))
    lens = torch.randint(0, Nk + 1, (B,), generator=torch.Generator().manual_seed(N)).to(torch.int32)
    lens[0] = Nk
    for causal, x in ((True, None), (True, lens.cuda()), (False, lens.cuda())):
        out, lse = pa.sage_attn_shared_prefix(q, kp, vp, k, v, kv_lens=x, causal=causal, layout=layout, return_lse=True)
        want, wl, ob, lb = ref.shared_prefix(q, kp, vp, k, v, x, causal, 0.0, layout)
        ref.check("lse", lse, wl, lb)
        ref.check("out", out, want, ob)
