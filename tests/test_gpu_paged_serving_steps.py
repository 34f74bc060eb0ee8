"""The norms with rotation, the appends and the attention over pages together, as a serving program and a training step use them."""
import types

import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _cache(c):
    return dict(k_cache=c[0], v_cache=c[1], k_scale=c[2], v_scale=c[3])


@pytest.mark.parametrize("d,dt,window,sink", [(128, torch.bfloat16, 0, 0), (64, torch.float16, 70, 5), (256, torch.bfloat16, 40, 33)])
def test_a_prompt_and_steps_of_generation(d, dt, window, sink):
    """Prompts of different lengths in one padded call, then ragged steps of one to three tokens; pages are handed out as they are needed and, behind the
    window, taken back and given to others."""
    pa = _pa()
    B, H, Hkv, page, of_one, pages = 3, 8, 2, 32, 12, 22
    g = _gen(0)
    f = pa.sage_rope_frequencies(d, base=500000.0)
    w = [torch.randn(d, generator=g, device="cuda").mul_(0.2).add_(1.0) for _ in range(2)]
    cache = pref.new_cache(pages, Hkv, page, d)
    mirror = [t.clone() for t in cache]
    free, tbl, lens = list(range(pages))[::-1], [[-1] * of_one for _ in range(B)], [0] * B
    for step in range(14):
        counts = [150, 33, 1] if step == 0 else torch.randint(0, 4, (B,), generator=torch.Generator().manual_seed(step)).tolist()
        N = max(max(counts), 1)
        for b in range(B):
            lens[b] += counts[b]
            for i in range(of_one):
                if 32 * i < lens[b] and tbl[b][i] < 0 and not (window and 32 * i >= sink and 32 * i + 32 <= lens[b] - counts[b] - window):
                    tbl[b][i] = free.pop()
                if window and tbl[b][i] >= 0 and 32 * i >= sink and 32 * i + 32 <= lens[b] - max(counts[b], 1) + 1 - window:      # (seen by no query from here on)
                    free.append(tbl[b][i])
                    tbl[b][i] = -1
        x = torch.randn((B, N, H + 2 * Hkv, d), generator=g, device="cuda").to(dt)          # a fused projection
        q, k, v = x.split([H, Hkv, Hkv], dim=2)
        tl, cl, t = _int(lens), _int(counts), torch.tensor(tbl, dtype=torch.int32, device="cuda")
        pos = (tl - cl)[:, None] + torch.arange(N, dtype=torch.int32, device="cuda")
        qr, kr = pa.sage_qk_norm_rope(q, k, f, *w, positions=pos, layout="NHD")
        ref.check("q", qr, *pref.norm_rope(q, w[0], f, pos, 1e-6, False, 1.0, "NHD"))
        ref.check("k", kr, *pref.norm_rope(k, w[1], f, pos, 1e-6, False, 1.0, "NHD"))
        want = pref.append(kr, mirror[0], mirror[2], t, tl, cl, "NHD") + pref.append(v, mirror[1], mirror[3], t, tl, cl, "NHD")
        pa.sage_cache_append(kr, v, *cache, t, kv_lens=tl, new_lens=cl, layout="NHD")
        for name, got, exp in zip(("k codes", "k scale", "v codes", "v scale"), (cache[0], cache[2], cache[1], cache[3]), want):
            pref.same(f"{name} of step {step}", got, exp)
        mirror = [y.clone() for y in cache]
        out, lse = pa.sage_attn_paged(qr.contiguous(), **_cache(cache), page_table=t, kv_lens=tl, q_lens=cl, window=window, sink=sink, layout="NHD", return_lse=True)
        o, l, ob, lb = pref.paged(qr, dict(_cache(cache), page_table=t), tl, cl, True, window, sink, 0.0, "NHD")
        ref.check(f"lse of step {step}", lse, l, lb)
        ref.check(f"output of step {step}", out, o, ob)
    assert lens[0] > 150 and (not window or -1 in tbl[0][:4])


def test_attention_over_8_bits_is_near_that_over_16():
    """A prompt attended to from the cache it was appended to, against the 16-bit attention of the same tokens: codes are off by 2^-4 of a value."""
    pa = _pa()
    g = _gen(4)
    k, v, q = (torch.randn((2, h, n, 128), generator=g, device="cuda").bfloat16() for h, n in ((2, 700), (2, 700), (8, 5)))
    cache, tbl = pref.new_cache(25, 2, 64, 128), pref.table(2, 704, 64, 25)
    lens = _int([700, 700])
    pa.sage_cache_append(k, v, *cache, tbl, kv_lens=lens)
    got = pa.sage_attn_paged(q, **_cache(cache), page_table=tbl, kv_lens=lens)
    want = pa.sage_attn_shared_prefix(q, None, None, k, v)
    # A code is off by 2^-4 of its value at most, 2^-4 / sqrt(3) = 0.036 in the root mean square of steps met evenly.  So are the values; a score of unit normals is off by
    # 0.036 |q| / sqrt(d) sqrt(d) = 0.036 then, and a weight by that share of itself.  Together 0.051 of an output, whose cosine with the exact one is 1 - 0.051^2 / 2 > 0.998 on
    # average; single rows spread, hence the room.
    cos = torch.nn.functional.cosine_similarity(got.double().flatten(2), want.double().flatten(2), dim=-1)
    assert cos.min() > 0.97


def test_steps_captured_into_two_graphs_that_share_a_workspace():
    pa = _pa()
    B, H, Hkv, d, page, of_one = 2, 8, 2, 128, 64, 40
    f = pa.sage_rope_frequencies(d)
    w = [torch.ones(d, device="cuda") for _ in range(2)]
    pages = B * of_one
    tbl, lens = pref.table(B, page * of_one, page, pages), _int([2000, 1500])
    sides = []
    c = pref.filled(B, Hkv, page * of_one, page, d, torch.bfloat16, spare=0)
    room = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    for side in range(3):                                  # two graphs and an eager twin
        s = types.SimpleNamespace(x=torch.zeros((B, 1, H + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda"), cache=[c[n].clone() for n in ("k_cache", "v_cache", "k_scale", "v_scale")])
        s.q, s.k = torch.empty((B, 1, H, d), dtype=torch.bfloat16, device="cuda"), torch.empty((B, 1, Hkv, d), dtype=torch.bfloat16, device="cuda")
        s.out, s.pos = torch.empty_like(s.q), torch.zeros((B, 1), dtype=torch.int32, device="cuda")
        def step(s=s):
            pa.sage_qk_norm_rope(s.x[:, :, :H], s.x[:, :, H:H + Hkv], f, *w, positions=s.pos, layout="NHD", q_out=s.q, k_out=s.k)
            pa.sage_cache_append(s.k, s.x[:, :, H + Hkv:], *s.cache, tbl, kv_lens=lens, layout="NHD")
            pa.sage_attn_paged(s.q, **_cache(s.cache), page_table=tbl, kv_lens=lens, layout="NHD", out=s.out, workspace=room)
        s.step = step
        sides.append(s)
    for s in sides[:2]:
        s.step()
        torch.cuda.synchronize()
        s.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s.graph):
            s.step()
    sides[2].step()
    for i in range(4):
        lens += 1
        x = torch.randn(sides[0].x.shape, generator=_gen(i), device="cuda").bfloat16()
        for s in sides:
            s.x.copy_(x)
            s.pos.copy_(lens[:, None] - 1)
        sides[i % 2].graph.replay()
        sides[2].step()
        sides[1 - i % 2].graph.replay()
        torch.cuda.synchronize()
        for s in sides[:2]:
            assert torch.equal(s.out, sides[2].out)
            for a, b in zip(s.cache, sides[2].cache):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_two_streams_at_once():
    pa = _pa()
    c = [pref.filled(4, 2, 4096, 64, 128, torch.bfloat16, seed=s) for s in range(2)]
    q = [torch.randn((4, 8, 1, 128), generator=_gen(s), device="cuda").bfloat16() for s in range(2)]
    want = [pa.sage_attn_paged(q[s], **c[s], return_lse=True) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[pa.sage_attn_paged(q[s], **c[s], return_lse=True, stream=streams[s]) for s in range(2)] for _ in range(10)]
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for turn in got:
        for s in range(2):
            assert torch.equal(turn[s][0], want[s][0]) and torch.equal(turn[s][1], want[s][1])


def test_a_pool_larger_than_32_bits_of_bytes():
    """Pages at both ends of a pool of 4.5 GB a tensor."""
    pa = _pa()
    Hkv, page, d, pages = 8, 64, 128, 68000
    cache = [torch.empty((pages, Hkv, page, d), dtype=torch.uint8, device="cuda").view(pref.E4M3) for _ in range(2)]
    cache += [torch.empty((pages, Hkv, page // 32), dtype=torch.uint8, device="cuda").view(pref.E8M0) for _ in range(2)]
    at = [0, 67999, 65536, 32768, 65535, 1]
    tbl, lens = _int([at[:3], at[3:]]), _int([180, 129])
    small, stbl = pref.new_cache(6, Hkv, page, d), _int([[0, 1, 2], [3, 4, 5]])
    g = _gen(7)
    k, v = (torch.randn((2, Hkv, 180, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((2, 16, 2, d), generator=g, device="cuda").bfloat16()
    for c, t in ((cache, tbl), (small, stbl)):
        pa.sage_cache_append(k, v, *c, t, kv_lens=lens, new_lens=lens)
    got = pa.sage_attn_paged(q, **_cache(cache), page_table=tbl, kv_lens=lens, return_lse=True)
    want = pa.sage_attn_paged(q, **_cache(small), page_table=stbl, kv_lens=lens, return_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for n, i in enumerate(at):
        for big, little in zip(cache, small):
            tokens = min(max(int(lens[n // 3]) - 64 * (n % 3), 0), 64)
            if big.dim() == 4:
                assert torch.equal(big[i, :, :tokens].view(torch.uint8), little[n, :, :tokens].view(torch.uint8))


def test_a_training_step_learns_the_weights_of_the_norms():
    """The gradient goes through a step of descent in float32 as that of the definition in float64 does."""
    pa = _pa()
    g = _gen(2)
    B, H, N, d = 2, 4, 60, 64
    f, pos = pa.sage_rope_frequencies(d), torch.arange(N, device="cuda")
    q, k, tq, tk = (torch.randn((B, H, N, d), generator=g, device="cuda").bfloat16() for _ in range(4))
    w = [torch.ones(d, device="cuda") for _ in range(2)]
    for step in range(3):
        yq, yk = pa.sage_qk_norm_rope(q, k, f, *w)
        dyq, dyk = (yq - tq), (yk - tk)                 # of half the squared distance
        dq, dk, dqw, dkw = pa.sage_qk_norm_rope_bwd(dyq, q, dyk, k, f, *w)
        for x, dy, wt, dx, dw in ((q, dyq, w[0], dq, dqw), (k, dyk, w[1], dk, dkw)):
            want, bound, want_w, bound_w = pref.norm_rope_bwd(dy, x, wt, f, pos, 1e-6, False, 1.0, "HND")
            ref.check("dx", dx, want, bound)
            ref.check("dw", dw, want_w, bound_w)
        w = [w[0] - 1e-3 * dqw, w[1] - 1e-3 * dkw]


def test_a_stream_of_another_gpu_and_tensors_that_do_not_go_together():
    """(One GPU is enough: the stream says that it is the next one's, and its handle is the default stream's.)"""
    pa = _pa()
    other = types.SimpleNamespace(cuda_stream=0, device_index=torch.cuda.current_device() + 1)
    c = pref.filled(2, 2, 64, 32, 64, torch.bfloat16)
    cache = [c[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")]
    before = [t.view(torch.uint8).clone() for t in cache]
    q, k = torch.ones((2, 4, 1, 64), device="cuda").bfloat16(), torch.ones((2, 2, 1, 64), device="cuda").bfloat16()
    f, w = pa.sage_rope_frequencies(64), torch.ones(64, device="cuda")
    for call in (lambda **kw: pa.sage_qk_norm_rope(q, k, f, w, w, **kw), lambda **kw: pa.sage_qk_norm_rope_bwd(q, q, k, k, f, w, w, **kw),
                 lambda **kw: pa.sage_cache_append(k, k, *cache, c["page_table"], **kw), lambda **kw: pa.sage_attn_paged(q, **c, **kw)):
        with pytest.raises(ValueError, match="stream"):
            call(stream=other)
    bad = [
        (ValueError, lambda: pa.sage_qk_norm_rope(q.cpu(), None, f)), (TypeError, lambda: pa.sage_qk_norm_rope(q.float(), None, f)), (ValueError, lambda: pa.sage_qk_norm_rope(q, k[:1], f)),
        (ValueError, lambda: pa.sage_qk_norm_rope(q, k.float(), f)), (ValueError, lambda: pa.sage_qk_norm_rope(q, None, f, k_weight=w)), (ValueError, lambda: pa.sage_qk_norm_rope(q, None, f, w[:32])),
        (TypeError, lambda: pa.sage_qk_norm_rope(q, k, f, w, w.bfloat16())), (TypeError, lambda: pa.sage_qk_norm_rope(q, k, f, w.half())), (TypeError, lambda: pa.sage_qk_norm_rope(q, k, f.float())),
        (ValueError, lambda: pa.sage_qk_norm_rope(q, k, f, positions=torch.zeros(3, dtype=torch.int32, device="cuda"))), (ValueError, lambda: pa.sage_qk_norm_rope(q[0], None, f)),
        (ValueError, lambda: pa.sage_qk_norm_rope(q, None, f, k_out=k)), (ValueError, lambda: pa.sage_qk_norm_rope(q, k, f, q_out=k)), (pa.SageError, lambda: pa.sage_qk_norm_rope(q, k, f, eps=-1.0)),
        (ValueError, lambda: pa.sage_qk_norm_rope_bwd(k, q, None, None, f)), (ValueError, lambda: pa.sage_qk_norm_rope_bwd(q, q, None, k, f)),
        (ValueError, lambda: pa.sage_qk_norm_rope_bwd(q, q, None, None, f, dq_weight=w)), (ValueError, lambda: pa.sage_qk_norm_rope_bwd(q, q, k, k, f, dk=q)),
        (ValueError, lambda: pa.sage_cache_append(k, k[:1], *cache, c["page_table"])), (ValueError, lambda: pa.sage_cache_append(q, q, *cache, c["page_table"])),
        (TypeError, lambda: pa.sage_cache_append(k, k, cache[0].view(torch.uint8), *cache[1:], c["page_table"])), (ValueError, lambda: pa.sage_cache_append(k, k, *cache, c["page_table"][:1])),
        (TypeError, lambda: pa.sage_cache_append(k, k, *cache[:2], cache[2].view(torch.uint8), cache[3], c["page_table"])),
        (TypeError, lambda: pa.sage_cache_append(k, k, *cache, c["page_table"].long())), (ValueError, lambda: pa.sage_cache_append(k, k, *cache, c["page_table"], kv_lens=_int([1]))),
        (ValueError, lambda: pa.sage_cache_append(k, k, *cache[:3], cache[3][:1], c["page_table"])), (ValueError, lambda: pa.sage_cache_append(k, k, *cache, c["page_table"][0])),
        (ValueError, lambda: pa.sage_attn_paged(q[:1], **c)), (ValueError, lambda: pa.sage_attn_paged(torch.ones((2, 3, 4, 64), device="cuda").bfloat16().transpose(1, 2), **c)), (TypeError, lambda: pa.sage_attn_paged(q.float(), **c)),
        (ValueError, lambda: pa.sage_attn_paged(q, **c, out=k)), (pa.SageError, lambda: pa.sage_attn_paged(q, **c, window=-1)), (pa.SageError, lambda: pa.sage_attn_paged(q, **c, sink=-1)),
        (pa.SageError, lambda: pa.sage_attn_paged(q, **c, window=5, causal=False)), (pa.SageError, lambda: pa.sage_attn_paged(torch.ones((2, 3, 1, 64), device="cuda").bfloat16(), **c)),
        (pa.SageError, lambda: pa.sage_attn_paged(q, **c, window=2 ** 40 * -1)), (ValueError, lambda: pa.sage_attn_paged(q, **c, q_lens=_int([1, 1, 1]))),
        (pa.SageError, lambda: pa.sage_attn_paged(q, **c, sm_scale=float("nan"))), (pa.SageError, lambda: pa.sage_qk_norm_rope(q, k, f, scale=float("inf"))),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
    for t, was in zip(cache, before):
        assert torch.equal(t.view(torch.uint8), was)
