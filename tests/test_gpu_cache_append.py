"""New tokens into a cache of 8 bits and pages: bit for bit what the definition says."""
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


def _tokens(B, Hkv, N, d, dt, layout, seed=0, std=1.0, wide=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((B, Hkv, N, d), generator=g, device="cuda") * std
    if wide:
        x *= torch.exp2(torch.randint(-12, 5, (B, Hkv, N, 1), generator=g, device="cuda").float())        # tokens of very different sizes
    return ref.to_layout(x.to(dt), layout)


def _append(pa, k, v, cache, tbl, lens, news, layout="HND", **kw):
    print(f"append k={tuple(k.shape)} cache={tuple(cache[0].shape)} {k.dtype} {layout} lens={None if lens is None else lens.tolist()} "
          f"new={None if news is None else news.tolist()}", flush=True)
    want = pref.append(k, cache[0], cache[2], tbl, lens, news, layout) + pref.append(v, cache[1], cache[3], tbl, lens, news, layout)
    pa.sage_cache_append(k, v, cache[0], cache[1], cache[2], cache[3], tbl, kv_lens=lens, new_lens=news, layout=layout, **kw)
    torch.cuda.synchronize()
    for name, got, exp in zip(("k codes", "k scale", "v codes", "v scale"), (cache[0], cache[2], cache[1], cache[3]), want):
        pref.same(name, got, exp)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,Hkv,N,cap,page", [(1, 1, 1, 32, 32), (2, 2, 5, 128, 64), (3, 1, 31, 96, 96), (2, 3, 33, 160, 32), (1, 2, 200, 256, 128), (5, 4, 1, 64, 32)])
def test_sizes(B, Hkv, N, cap, page, d):
    """Into an empty cache, and then step after step behind what is there, up to the end of the table."""
    pa = _pa()
    dt, layout = (torch.bfloat16, "HND") if (B + N + d // 64) % 2 else (torch.float16, "NHD")
    pages = B * (cap // page) + 2
    cache, tbl = pref.new_cache(pages, Hkv, page, d), pref.table(B, cap, page, pages)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    for step in range(4):
        n = N if step == 0 else (N + step) % 7 + 1
        if int(lens.max()) + n > cap:
            break
        lens += n
        k, v = (_tokens(B, Hkv, n, d, dt, layout, seed=10 * step + s) for s in range(2))
        _append(pa, k, v, cache, tbl, lens, None, layout)


def test_ragged_new_tokens_and_lengths_out_of_range():
    pa = _pa()
    cache, tbl = pref.new_cache(30, 2, 64, 128), pref.table(7, 256, 64, 30)
    k, v = (_tokens(7, 2, 40, 128, torch.bfloat16, "NHD", seed=s) for s in range(2))
    #                none     negative  all    one      more new than there are   past the table   more than N
    _append(pa, k, v, cache, tbl, _int([100, 90, 256, 33, 17, 5000, 70]), _int([0, -3, 40, 1, 25, 40, 1000]), "NHD")
    _append(pa, k, v, cache, tbl, None, None, "NHD")
    _append(pa, k, v, cache, tbl, _int([-5, 0, 0, 1, 2, 3, 4]), None, "NHD")


def test_pages_that_are_none_are_left_out():
    pa = _pa()
    cache, tbl = pref.new_cache(12, 2, 32, 64), pref.table(3, 128, 32, 12)
    tbl[0, 1], tbl[1, 0], tbl[2, 3] = -1, 12, 2 ** 31 - 1
    k, v = (_tokens(3, 2, 100, 64, torch.float16, "HND", seed=s) for s in range(2))
    _append(pa, k, v, cache, tbl, _int([110, 128, 101]), None)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_a_scale_that_rises_and_one_that_stays(dt):
    pa = _pa()
    cache, tbl = pref.new_cache(4, 2, 32, 64), pref.table(1, 32, 32, 4)
    lens = _int([0])
    for i, std in enumerate((1.0, 1e-3, 30.0, 0.1, 900.0, 1e-6, 2000.0)):
        lens += 3
        k, v = (_tokens(1, 2, 3, 64, dt, "HND", seed=i + 50 * s, std=std, wide=False) for s in range(2))
        _append(pa, k, v, cache, tbl, lens, None)
    # taken back by five tokens and written again: the scale stays
    lens -= 5
    lens += 2
    k, v = (_tokens(1, 2, 2, 64, dt, "HND", seed=99 + s, std=0.01, wide=False) for s in range(2))
    _append(pa, k, v, cache, tbl, lens, None)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_the_ends_of_the_type(dt):
    """The largest values, the smallest, zeros of both signs, borders of a scale, ties, infinities and NaN."""
    pa = _pa()
    info = torch.finfo(dt)
    rows = []
    for x in (info.max, -info.max, 448.0, 449.0, 447.0, 447.9, 448.0 * 2 ** -20, info.tiny, info.smallest_normal / 4, 0.0, -0.0, 57344.0 if dt == torch.float16 else 2.0 ** 127):
        row = torch.zeros(64, dtype=torch.float64)
        row[3], row[4], row[5] = x, -x / 3, x / 2 ** 17
        rows.append(row)
    ties = torch.zeros(64, dtype=torch.float64)
    ties[:16], ties[16:32], ties[63] = 256 + 8 * torch.arange(16), 2.0 ** -9 * torch.arange(16) / 2, 448
    rows.append(ties)
    for bad in (math.inf, -math.inf, math.nan):
        row = torch.linspace(-3, 3, 64, dtype=torch.float64)
        row[10] = bad
        rows.append(row)
    only = torch.full((64,), math.inf, dtype=torch.float64)
    rows.append(only)
    for row in rows:                                     # alone in a block, and behind an ordinary token
        for before in (0, 1):
            x = row.to(dt).reshape(1, 1, 1, 64).cuda()
            cache, tbl = pref.new_cache(2, 1, 32, 64), pref.table(1, 32, 32, 2)
            if before:
                one = _tokens(1, 1, 1, 64, dt, "HND", wide=False)
                pa.sage_cache_append(one, one, *cache, tbl, kv_lens=_int([1]))
            _append(pa, x, x.flip(-1).contiguous(), cache, tbl, _int([1 + before]), None)


@pytest.mark.parametrize("shift", [1, 8])
def test_views(shift):
    """New tokens as slices of a fused projection, aligned to a vector or not."""
    pa = _pa()
    B, Hkv, N, d = 3, 2, 21, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    big = torch.randn((B, N, 4 * Hkv, d + shift), generator=g, device="cuda").bfloat16()
    k, v = big[:, :, Hkv:2 * Hkv, shift:], big[:, :, 3 * Hkv:, :d]
    cache, tbl = pref.new_cache(7, Hkv, 32, d), pref.table(B, 64, 32, 7)
    _append(pa, k, v, cache, tbl, _int([21, 30, 64]), None, "NHD")
    _append(pa, k.transpose(1, 2), v.transpose(1, 2), cache, tbl, _int([42, 33, 64]), _int([21, 3, 0]), "HND")


def test_what_is_not_written_stays():
    """Pages that no new token goes to, codes behind the last token, other blocks' scales: every byte."""
    pa = _pa()
    cache, tbl = pref.new_cache(9, 2, 64, 64, fill=0x55), pref.table(2, 192, 64, 9)
    before = [t.view(torch.uint8).clone() for t in cache]
    k, v = (_tokens(2, 2, 20, 64, torch.bfloat16, "HND", seed=s) for s in range(2))
    pa.sage_cache_append(k, v, *cache, tbl, kv_lens=_int([20, 100]))
    torch.cuda.synchronize()
    touched = torch.zeros((9, 64), dtype=torch.bool)
    blocks = torch.zeros((9, 2), dtype=torch.bool)
    for b, (lo, hi) in enumerate(((0, 20), (80, 100))):
        for t in range(lo, hi):
            touched[int(tbl[b, t // 64]), t % 64] = True
            blocks[int(tbl[b, t // 64]), t % 64 // 32] = True
    # (the block that token 80 is in starts at 64: its 16 earlier tokens may be rounded again)
    for t in range(64, 80):
        touched[int(tbl[1, t // 64]), t % 64] = True
    for now, was in zip(cache[:2], before[:2]):
        assert torch.equal(now.view(torch.uint8).transpose(1, 2)[~touched.cuda()], was.transpose(1, 2)[~touched.cuda()])
    for now, was in zip(cache[2:], before[2:]):
        assert torch.equal(now.view(torch.uint8).transpose(1, 2)[~blocks.cuda()], was.transpose(1, 2)[~blocks.cuda()])


def test_captured_steps():
    pa = _pa()
    cache, tbl = pref.new_cache(5, 2, 32, 128), pref.table(2, 64, 32, 5)
    other = [t.clone() for t in cache]
    lens = _int([0, 7])
    k, v = (_tokens(2, 2, 1, 128, torch.bfloat16, "HND", seed=s) for s in range(2))
    pa.sage_cache_append(_tokens(2, 2, 7, 128, torch.bfloat16, "HND"), _tokens(2, 2, 7, 128, torch.bfloat16, "HND"), *cache, tbl, kv_lens=lens, new_lens=_int([0, 7]))
    for a, b in zip(other, cache):
        a.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.sage_cache_append(k, v, *cache, tbl, kv_lens=lens)
    for step in range(4):
        lens += 1
        k.copy_(_tokens(2, 2, 1, 128, torch.bfloat16, "HND", seed=30 + step))
        graph.replay()
        pa.sage_cache_append(k, v, *other, tbl, kv_lens=lens)
        torch.cuda.synchronize()
        for a, b in zip(cache, other):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
