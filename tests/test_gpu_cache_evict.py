"""Eviction from a cache: which tokens stay, and that rows, weights and lengths follow - all of it exactly."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _check(pa, w, keep, sink, recent, lens=None, d=64, dt=torch.bfloat16, layout="HND", seed=0):
    B, Hkv, nk = w.shape
    print(f"evict B={B} Hkv={Hkv} {nk} -> {keep} sink={sink} recent={recent} d={d} {layout} lens={None if lens is None else lens.tolist()}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, v = (ref.to_layout(torch.randn((B, Hkv, nk, d), generator=g, device="cuda").to(dt), layout) for _ in range(2))
    rows = (B, keep, Hkv, d) if layout == "NHD" else (B, Hkv, keep, d)
    outs = dict(k_out=torch.full(rows, 5.0, dtype=dt, device="cuda"), v_out=torch.full(rows, 6.0, dtype=dt, device="cuda"),
                weights_out=torch.full((B, Hkv, keep), 7.0, device="cuda"), kept=torch.full((B, Hkv, keep), -8, dtype=torch.int32, device="cuda"),
                lens_out=torch.full((B,), -9, dtype=torch.int32, device="cuda"))
    ko, vo, wo, kept, left = pa.sage_cache_evict(k, v, w, keep, sink=sink, recent=recent, kv_lens=lens, layout=layout, **outs)
    torch.cuda.synchronize()
    want = ref.evict(k, v, w, keep, sink, recent, lens, layout)
    ko, vo, kh, vh = (ref.heads_first(x, layout) for x in (ko, vo, k, v))
    for b in range(B):
        n = len(want[b][0])
        assert left[b].item() == n
        for h in range(Hkv):
            assert kept[b, h, :n].tolist() == want[b][h], (b, h)
            at = torch.tensor(want[b][h], device="cuda", dtype=torch.long)
            assert torch.equal(ko[b, h, :n], kh[b, h][at]) and torch.equal(vo[b, h, :n], vh[b, h][at])
            assert torch.equal(wo[b, h, :n].view(torch.int32), w[b, h][at].view(torch.int32))
            assert (ko[b, h, n:] == 5).all() and (vo[b, h, n:] == 6).all() and (wo[b, h, n:] == 7).all() and (kept[b, h, n:] == -8).all()


def _w(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(2.0).exp_()


@pytest.mark.parametrize("nk,keep,sink,recent", [(1, 1, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (2, 1, 0, 1), (63, 20, 4, 7), (64, 64, 0, 64), (65, 64, 0, 64),
                                                 (700, 256, 4, 32), (700, 256, 0, 256), (1024, 1023, 0, 0), (1025, 1, 0, 0), (5000, 1700, 1, 3),
                                                 (5000, 10, 5, 5), (20000, 9999, 4, 100)])
def test_sizes(nk, keep, sink, recent):
    pa = _pa()
    _check(pa, _w((2, 3, nk), nk), keep, sink, recent)


@pytest.mark.parametrize("layout", ["HND", "NHD"])
def test_more_than_the_caches_hold(layout):
    """A call that moves over 256 MB."""
    pa = _pa()
    lens = torch.tensor([40003, 20000], dtype=torch.int32, device="cuda")
    _check(pa, _w((2, 4, 40003), 3), 33001, 4, 100, lens, d=128, layout=layout)


@pytest.mark.parametrize("d,dt,layout", [(64, torch.float16, "NHD"), (128, torch.bfloat16, "NHD"), (128, torch.float16, "HND"), (256, torch.bfloat16, "HND"),
                                         (256, torch.float16, "NHD")])
def test_widths_types_and_layouts(d, dt, layout):
    pa = _pa()
    lens = torch.tensor([777, 300, 0, 301, 1, 2000], dtype=torch.int32, device="cuda")     # (the last one is cut to the capacity)
    _check(pa, _w((6, 2, 777), d), 300, 3, 50, lens, d, dt, layout)


def test_more_room_than_tokens():
    pa = _pa()
    _check(pa, _w((2, 2, 100), 1), 150, 4, 60)


def test_ties_nan_and_signs():
    pa = _pa()
    w = torch.ones((1, 8, 3000), device="cuda")
    w[0, 1] = 0.0
    w[0, 2, ::2] = -0.0                      # equal to zero
    w[0, 2, 1::2] = 0.0
    w[0, 3] = torch.arange(3000, device="cuda") % 7
    w[0, 4] = math.nan
    w[0, 4, 2000:2100] = -math.inf           # still more than a NaN
    w[0, 5, 1500:] = math.inf
    w[0, 6] = -torch.arange(3000, device="cuda").float()
    w[0, 7] = torch.arange(3000, device="cuda").float() * 1e-42          # subnormal numbers keep their order
    _check(pa, w, 1000, 0, 0)
    _check(pa, w, 1000, 10, 20)


def test_what_stands_behind_a_length_is_not_looked_at():
    pa = _pa()
    w = _w((2, 2, 500), 3)
    lens = torch.tensor([200, 333], dtype=torch.int32, device="cuda")
    for fill in (math.inf, math.nan):
        for b in range(2):
            w[b, :, lens[b].item():] = fill
        _check(pa, w, 100, 2, 9, lens)


def test_long_rows_another_stream_and_replays():
    pa = _pa()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    B, Hkv, nk, keep, d = 1, 2, 150001, 70000, 64
    k, v = (torch.randn((B, Hkv, nk, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randint(0, 40000, (B, Hkv, nk), generator=g, device="cuda").float()          # many ties
    lens = torch.tensor([nk], dtype=torch.int32, device="cuda")
    order = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep].sort(-1).values
    want = k.gather(2, order[..., None].expand(-1, -1, -1, d))
    outs = pa.sage_cache_evict(k, v, w, keep, kv_lens=lens)
    assert torch.equal(outs[3].long(), order) and torch.equal(outs[0], want) and torch.equal(outs[2], w.gather(-1, order))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = pa.sage_cache_evict(k, v, w, keep, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(outs, other))
    kw = dict(k_out=torch.zeros_like(outs[0]), v_out=torch.zeros_like(outs[1]), weights_out=torch.zeros_like(outs[2]), kept=torch.zeros_like(outs[3]),
              lens_out=torch.zeros_like(outs[4]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.sage_cache_evict(k, v, w, keep, sink=3, recent=9, kv_lens=lens, **kw)
    for n in (nk, 100000, 70000, 60000):
        lens.fill_(n)
        w.add_(0.0).copy_(w.flip(-1))
        graph.replay()
        again = pa.sage_cache_evict(k, v, w, keep, sink=3, recent=9, kv_lens=lens)
        torch.cuda.synchronize()
        n = min(n, keep)
        assert torch.equal(kw["lens_out"], again[4])
        assert all(torch.equal(kw[x][:, :, :n], again[i][:, :, :n]) for i, x in enumerate(("k_out", "v_out", "weights_out", "kept")))


@pytest.mark.parametrize("layout", ["HND", "NHD"])
def test_room_for_more_than_is_kept(layout):
    """A cache cut into one of the same size: places behind what is kept stay as they were."""
    pa = _pa()
    B, Hkv, nk, d, keep = 3, 2, 500, 128, 200
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    k, v = (ref.to_layout(torch.randn((B, Hkv, nk, d), generator=g, device="cuda").half(), layout) for _ in range(2))
    w, lens = _w((B, Hkv, nk), 6), torch.tensor([500, 150, 333], dtype=torch.int32, device="cuda")
    want = ref.evict(k, v, w, keep, 4, 50, lens, layout)
    old = dict(k_out=torch.full_like(k, 5.0), v_out=torch.full_like(v, 6.0), weights_out=torch.full_like(w, 7.0))
    for room, outs in ((nk, old), (nk, {}), (201, {})):
        ko, vo, wo, kept, left = pa.sage_cache_evict(k, v, w, keep, sink=4, recent=50, kv_lens=lens, layout=layout, room=room, **outs)
        kh, vh, ko, vo = (ref.heads_first(x, layout) for x in (k, v, ko, vo))
        assert ko.shape == (B, Hkv, room, d) and wo.shape == (B, Hkv, room) and kept.shape == (B, Hkv, keep)
        for b in range(B):
            n = len(want[b][0])
            assert left[b].item() == n
            for h in range(Hkv):
                at = torch.tensor(want[b][h], device="cuda", dtype=torch.long)
                assert kept[b, h, :n].tolist() == want[b][h]
                assert torch.equal(ko[b, h, :n], kh[b, h][at]) and torch.equal(vo[b, h, :n], vh[b, h][at]) and torch.equal(wo[b, h, :n], w[b, h][at])
                for x, y in ((ko, 5.0), (vo, 6.0), (wo, 7.0)):
                    assert (x[b, h, n:] == (y if outs else 0.0)).all()
