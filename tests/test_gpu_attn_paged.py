"""Attention over a cache of 8 bits and pages, against float64."""
import math

import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _q(B, H, N, d, dt, layout, seed=0, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    return ref.to_layout(torch.randn((B, H, N, d), generator=g, device="cuda").mul_(std).to(dt), layout)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _check(pa, q, c, lens=None, q_lens=None, causal=True, window=0, sink=0, sm_scale=0.0, layout="HND", **kw):
    print(f"paged q={tuple(q.shape)} cache={tuple(c['k_cache'].shape)} table={tuple(c['page_table'].shape)} {q.dtype} {layout} lens={None if lens is None else lens.tolist()} "
          f"q_lens={None if q_lens is None else q_lens.tolist()} causal={causal} window={window} sink={sink}", flush=True)
    out, lse = pa.sage_attn_paged(q, **c, kv_lens=lens, q_lens=q_lens, causal=causal, window=window, sink=sink, sm_scale=sm_scale, layout=layout, return_lse=True, **kw)
    torch.cuda.synchronize()
    want, wl, ob, lb = pref.paged(q, c, lens, q_lens, causal, window, sink, sm_scale, layout)
    ref.check("lse", lse, wl, lb)
    ref.check("out", out, want, ob)
    return out, lse


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,Hkv,N,cap,page", [(1, 1, 1, 1, 32, 32), (2, 2, 1, 1, 64, 64), (2, 4, 2, 1, 96, 32), (3, 8, 2, 1, 448, 64), (2, 4, 4, 5, 192, 96), (5, 8, 1, 3, 640, 128),
                                                (2, 6, 2, 33, 160, 32), (1, 8, 1, 40, 1024, 256), (2, 2, 2, 130, 384, 64), (2, 16, 8, 1, 2048, 64), (1, 4, 1, 300, 320, 32)])
def test_sizes(B, H, Hkv, N, cap, page, d):
    pa = _pa()
    dt, layout = (torch.bfloat16, "HND") if (B + N + d // 64) % 2 else (torch.float16, "NHD")
    c = pref.filled(B, Hkv, cap, page, d, dt)
    q = _q(B, H, N, d, dt, layout)
    _check(pa, q, c, layout=layout)
    lens = torch.randint(0, cap + 1, (B,), generator=torch.Generator().manual_seed(N)).to(torch.int32)
    lens[0] = cap - 1
    lens = lens.cuda()
    _check(pa, q, c, lens=lens, layout=layout)
    _check(pa, q, c, lens=lens, causal=False, sm_scale=0.03, layout=layout)
    counts = torch.randint(0, N + 1, (B,), generator=torch.Generator().manual_seed(N + 1)).to(torch.int32).cuda()
    _check(pa, q, c, lens=lens, q_lens=counts, layout=layout)
    for window, sink in ((1, 0), (2, 1), (31, 4), (32, 0), (33, 33), (100, 64), (10 ** 9, 5)):
        _check(pa, q, c, lens=lens, window=window, sink=sink, layout=layout)
    _check(pa, q, c, lens=lens, q_lens=counts, window=40, sink=3, layout=layout)


def test_lengths_around_the_tiles():
    """One token more and less than blocks, tiles and pages, none at all, and lengths out of range."""
    pa = _pa()
    lens = [0, 1, 31, 32, 33, 63, 64, 65, 95, 96, 127, 128, 129, 255, 256, 257, 511, 512, -3, 100000]
    for page, N in ((32, 1), (96, 2), (256, 1)):
        c = pref.filled(len(lens), 2, 768, page, 128, torch.bfloat16)
        q = _q(len(lens), 4, N, 128, torch.bfloat16, "HND")
        out, lse = _check(pa, q, c, lens=_int(lens))
        assert (out[0] == 0).all() and (out[18] == 0).all() and (lse[0] == -math.inf).all()
        for window, sink in ((33, 0), (200, 7)):
            _check(pa, q, c, lens=_int(lens), window=window, sink=sink)


@pytest.mark.parametrize("rows", [(4, 4), (5, 4), (8, 4), (9, 4), (16, 4), (17, 4), (33, 4), (1, 33), (7, 19)])
def test_rows_around_the_tiles(rows):
    """N G rows of a KV head: one wavefront's 32, two, a workgroup's 128, several; heads and queries that do not divide."""
    pa = _pa()
    N, G = rows
    c = pref.filled(2, 2, 512, 32, 64, torch.bfloat16)
    q = _q(2, 2 * G, N, 64, torch.bfloat16, "HND", seed=N)
    _check(pa, q, c, lens=_int([500, 77]), window=60, sink=5)
    _check(pa, q, c, lens=_int([500, 3]))


def test_what_is_not_seen_is_not_read():
    """NaN, and numbers of no page, in all places that no query sees: behind the last token and behind the window."""
    pa = _pa()
    for d, layout in ((64, "HND"), (128, "NHD"), (256, "HND")):
        for N, window, sink in ((1, 0, 0), (3, 0, 0), (1, 50, 5), (4, 50, 37)):
            c = pref.filled(3, 2, 384, 32, d, torch.bfloat16)
            lens = _int([0, 201, 300])
            q = _q(3, 4, N, d, torch.bfloat16, layout)
            want = _check(pa, q, c, lens=lens, window=window, sink=sink, layout=layout)
            for b, n in enumerate(lens.tolist()):
                lowest = max(n - N, 0) + 1 - window if window else 0
                for t in range(384):
                    if t < n and (t >= lowest or t < sink):
                        continue
                    at = int(c["page_table"][b, t // 32])
                    for x in "kv":
                        c[x + "_cache"].view(torch.uint8)[at, :, t % 32] = 0x7f if t % 2 else 0xff
                for i in range(12):
                    if 32 * i >= n or (32 * i >= sink and 32 * i + 32 <= lowest):
                        at = int(c["page_table"][b, i])
                        for x in "kv":
                            c[x + "_scale"].view(torch.uint8)[at] = 0xff
                        c["page_table"][b, i] = (-1, 2 ** 31 - 1, c["k_cache"].shape[0])[i % 3]
            got = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window, sink=sink, layout=layout, return_lse=True)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_pages_that_are_none_hold_no_tokens():
    pa = _pa()
    c = pref.filled(3, 2, 512, 64, 128, torch.float16)
    c["page_table"][0, 3], c["page_table"][1, 0], c["page_table"][1, 5] = -1, 10 ** 9, -(2 ** 31)
    c["page_table"][2, :] = -1
    for N in (1, 6, 70):
        q = _q(3, 4, N, 128, torch.float16, "HND")
        out, lse = _check(pa, q, c, lens=_int([512, 500, 400]))
        assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
        _check(pa, q, c, lens=_int([250, 380, 400]), window=100, sink=40)


def test_a_page_of_several_sequences():
    pa = _pa()
    c = pref.filled(4, 2, 256, 64, 64, torch.bfloat16)
    c["page_table"][1:, :2] = c["page_table"][0, :2]           # a shared prefix of two pages
    c["page_table"][3, 3] = c["page_table"][3, 0]              # and one twice in a sequence
    q = _q(4, 4, 2, 64, torch.bfloat16, "HND")
    _check(pa, q, c, lens=_int([256, 130, 200, 256]))


@pytest.mark.parametrize("N,G", [(1, 4), (5, 4), (40, 4), (130, 1)])
def test_nan_reaches_only_those_that_see_it(N, G):
    pa = _pa()
    for d in (64, 128, 256):
        for window, sink in ((0, 0), (37, 3)):
            c = pref.filled(2, 2, 256, 32, d, torch.bfloat16, seed=5)
            lens = _int([200, 131])
            q = _q(2, 2 * G, N, d, torch.bfloat16, "HND")
            for t, ch in ((199, 3), (185, d - 1), (170, 17), (2, 9), (60, 40)):
                at = int(c["page_table"][0, t // 32])
                c["v_cache"].view(torch.uint8)[at, 0, t % 32, ch] = 0xff if t % 2 else 0x7f
            _check(pa, q, c, lens=lens, window=window, sink=sink)
            at = int(c["page_table"][1, 130 // 32])                 # a key: whole rows, of those that see it
            c["k_cache"].view(torch.uint8)[at, 1, 130 % 32, 5] = 0x7f
            out, lse = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window, sink=sink, return_lse=True)
            assert out[1, G:, -1].isnan().all() and lse[1, G:, -1].isnan().all()
            assert not out[1, :G].isnan().any() and (N == 1 or not out[1, :, :-1].isnan().any())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_large_scores_and_scales_far_apart(dt):
    """A few keys take it all; blocks whose values differ by 2^40 (what fp16 holds of that); weights far below the largest."""
    pa = _pa()
    c = pref.filled(2, 2, 512, 32, 128, dt)
    _check(pa, _q(2, 4, 1, 128, dt, "HND", std=60.0), c)
    _check(pa, _q(2, 4, 9, 128, dt, "HND", std=0.01), c)
    lo = -20 if dt == torch.float16 else -60
    for x in "kv":
        s = c[x + "_scale"].view(torch.uint8)
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        e = torch.randint(lo, 6 if dt == torch.float16 else 60, s.shape, generator=g, device="cuda") if x == "v" else torch.randint(-20, -3, s.shape, generator=g, device="cuda")
        s.copy_((e + 127).to(torch.uint8))
    for N in (1, 50):
        _check(pa, _q(2, 4, N, 128, dt, "HND"), c, lens=_int([512, 77]))


@pytest.mark.parametrize("B,H,Hkv,cap,N", [(1, 8, 2, 40000, 1), (1, 2, 1, 20000, 40), (40, 8, 4, 1024, 1), (3, 32, 8, 9984, 2)])
def test_long_caches(B, H, Hkv, cap, N):
    """Keys of a query over several workgroups."""
    pa = _pa()
    page = 64
    cap = -(-cap // page) * page
    c = pref.filled(B, Hkv, cap, page, 128, torch.bfloat16)
    q = _q(B, H, N, 128, torch.bfloat16, "HND", std=2.0)
    lens = torch.linspace(cap, cap // 5, B).to(torch.int32).cuda()
    _check(pa, q, c, lens=lens)
    _check(pa, q, c, lens=lens, window=5000, sink=70)


@pytest.mark.parametrize("B,H,Hkv,N,cap,d,window,sink", [(64, 4, 4, 1, 4096, 128, 0, 0), (90, 8, 4, 3, 16384, 64, 4000, 40), (16, 16, 16, 140, 3008, 64, 0, 0), (64, 8, 4, 20, 2560, 128, 0, 0)])
def test_many_tiles_of_one_workgroup(B, H, Hkv, N, cap, d, window, sink):
    """More than the 16 whose places are looked up at a time: so many sequences that keys are not cut."""
    pa = _pa()
    c = pref.filled(B, Hkv, cap, 64, d, torch.bfloat16)
    c["page_table"][1, 20] = -1
    q = _q(B, H, N, d, torch.bfloat16, "HND")
    lens = torch.linspace(cap, cap // 3, B).to(torch.int32).cuda()
    some = [0, 1, B // 2, B - 1]                           # (every sequence is its own: the reference is asked for a few)
    out, lse = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window, sink=sink, return_lse=True)
    few = dict(c, page_table=c["page_table"][some])
    want, wl, ob, lb = pref.paged(q[some], few, lens[some], None, True, window, sink, 0.0, "HND")
    ref.check("lse", lse[some], wl, lb)
    ref.check("out", out[some], want, ob)
    alone = pa.sage_attn_paged(q, **c, kv_lens=lens, window=window, sink=sink)
    assert torch.equal(alone, out)


@pytest.mark.parametrize("N,G", [(1, 4), (6, 4), (70, 2)])
def test_scales_that_are_not_numbers(N, G):
    """A scale byte of 255, K's or V's: NaN in the rows that see its block, and in no others."""
    pa = _pa()
    for d in (64, 256):
        for x in ("k_scale", "v_scale"):
            c = pref.filled(2, 2, 320, 64, d, torch.bfloat16, seed=3)
            q = _q(2, 2 * G, N, d, torch.bfloat16, "HND")
            lens = _int([300, 200])
            clean = pa.sage_attn_paged(q, **c, kv_lens=lens, window=90, sink=3, return_lse=True)
            # block 8 (tokens 256 ..) of sequence 0, KV head 1
            c[x].view(torch.uint8)[int(c["page_table"][0, 4]), 1, 0] = 255
            got = pa.sage_attn_paged(q, **c, kv_lens=lens, window=90, sink=3, return_lse=True)
            pos = 300 - N + torch.arange(N, device="cuda")
            hit = torch.zeros((2, 2 * G, N), dtype=torch.bool, device="cuda")
            hit[0, G:] = (pos >= 256) & (pos - 90 < 287)
            assert hit.any() and (N < 50 or not hit[0, G].all())
            assert got[0][hit].isnan().all() and got[1][hit].isnan().all()
            assert torch.equal(got[0][~hit], clean[0][~hit]) and torch.equal(got[1][~hit], clean[1][~hit])


def test_values_beyond_fp16_with_small_weights():
    """A cache filled from bf16 tokens, read with fp16 queries: values far beyond 65504 whose weighted mean is within."""
    pa = _pa()
    for N in (1, 40):
        c = pref.filled(1, 1, 256, 32, 64, torch.float16, seed=8)
        e = c["v_scale"].view(torch.uint8)
        e[int(c["page_table"][0, 2])] = 127 + 14            # values of up to 448 2^14 in the block of tokens 64 .. 95
        c["v_cache"].view(torch.uint8)[int(c["page_table"][0, 2]), 0, 1:] = 0
        q = _q(1, 2, N, 64, torch.float16, "HND", std=0.02)      # (nearly equal weights: the one large token has some 2^-8)
        out, _ = _check(pa, q, c)
        assert out.isfinite().all() and out[:, :, -1].abs().max() > 5000


def test_rows_behind_the_last_query_stay():
    pa = _pa()
    for layout in ("HND", "NHD"):
        c = pref.filled(3, 2, 256, 64, 64, torch.float16)
        q = _q(3, 4, 6, 64, torch.float16, layout)
        lens, counts = _int([200, 64, 3]), _int([0, 4, 6])
        out = torch.full_like(q, 3.0)
        ref.heads_first(q, layout)[1, :, 4:] = math.nan        # queries that are not there
        got, lse = pa.sage_attn_paged(q, **c, kv_lens=lens, q_lens=counts, out=out, layout=layout, return_lse=True)
        torch.cuda.synchronize()
        assert got is out
        want, wl, ob, lb = pref.paged(q, c, lens, counts, True, 0, 0, 0.0, layout, out_was=torch.full_like(q, 3.0))
        ref.check("out", out, want, ob)
        ref.check("lse", lse, wl, lb)
        assert (ref.heads_first(out, layout)[1, :, 4:] == 3.0).all() and (ref.heads_first(out, layout)[0] == 3.0).all()


@pytest.mark.parametrize("N,cap", [(1, 64), (6, 256), (6, 4096), (50, 256), (50, 4096)])
def test_rows_behind_the_last_query_are_zeros_where_the_call_makes_the_output(N, cap):
    pa = _pa()
    for d, layout in ((64, "HND"), (256, "NHD")):
        c = pref.filled(4, 2, cap, 64, d, torch.bfloat16)
        q = _q(4, 6, N, d, torch.bfloat16, layout)
        lens, counts = _int([cap - 3, 64, 0, 7]), _int([N, 0, N, N // 2])
        junk = [torch.full_like(q, 9.0) for _ in range(3)] + [torch.full((4, 6, N), 9.0, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        del junk                                            # (what the allocator hands out next holds numbers)
        _check(pa, q, c, lens=lens, q_lens=counts, layout=layout)
        out = torch.full_like(q, 3.0)
        _, lse = pa.sage_attn_paged(q, **c, kv_lens=lens, q_lens=counts, out=out, layout=layout, return_lse=True)
        there = (torch.arange(N, device="cuda") < counts[:, None])[:, None]
        assert (ref.heads_first(out, layout)[~there.expand(4, 6, N)] == 3.0).all() and (lse[~there.expand(4, 6, N)] == 0).all()


def test_in_place_of_the_queries():
    pa = _pa()
    for N, cap in ((1, 64), (3, 4096)):
        c = pref.filled(2, 2, cap, 64, 128, torch.bfloat16)
        q = _q(2, 8, N, 128, torch.bfloat16, "HND")
        want = pa.sage_attn_paged(q, **c)
        got = pa.sage_attn_paged(q, **c, out=q)
        assert got is q and torch.equal(got, want)


def test_the_same_twice_and_on_a_stream():
    pa = _pa()
    c = pref.filled(3, 2, 4096, 64, 128, torch.bfloat16)
    q = _q(3, 8, 1, 128, torch.bfloat16, "HND")
    lens = _int([4096, 900, 2222])
    want = pa.sage_attn_paged(q, **c, kv_lens=lens, return_lse=True)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = pa.sage_attn_paged(q, **c, kv_lens=lens, return_lse=True, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    again = pa.sage_attn_paged(q, **c, kv_lens=lens, return_lse=True)
    for a, b, d in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, d)


def test_a_larger_workspace_and_a_small_one():
    pa = _pa()
    c = pref.filled(2, 2, 8192, 64, 128, torch.bfloat16)
    q = _q(2, 8, 1, 128, torch.bfloat16, "HND")
    want = pa.sage_attn_paged(q, **c)
    room = torch.full((1 << 26,), 0xff, dtype=torch.uint8, device="cuda")
    assert torch.equal(pa.sage_attn_paged(q, **c, workspace=room), want)
    with pytest.raises(pa.SageError):
        pa.sage_attn_paged(q, **c, workspace=room[:256])
