"""Eviction that sets the places behind the kept tokens to zeros itself."""
import ctypes

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _caches(B, Hkv, nk, d, layout, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, v = (ref.to_layout(torch.randn((B, Hkv, nk, d), generator=g, device="cuda").bfloat16(), layout) for _ in range(2))
    return k, v, torch.randn((B, Hkv, nk), generator=g, device="cuda").exp_()


def _expect(k, v, w, keep, sink, recent, lens, layout, outs):
    want = ref.evict(k, v, w, keep, sink, recent, lens, layout)
    ko, vo, wo, kept, left = outs
    ko, vo, kh, vh = (ref.heads_first(x, layout) for x in (ko, vo, k, v))
    for b in range(w.shape[0]):
        n = len(want[b][0])
        assert left[b].item() == n
        for h in range(w.shape[1]):
            at = torch.tensor(want[b][h], device="cuda", dtype=torch.long)
            assert kept[b, h, :n].tolist() == want[b][h]
            assert torch.equal(ko[b, h, :n], kh[b, h][at]) and torch.equal(vo[b, h, :n], vh[b, h][at]) and torch.equal(wo[b, h, :n], w[b, h][at])
            for x in (ko, vo, wo, kept):
                assert (x[b, h, n:] == 0).all()


# (one launch, and two: by the room, by the row's length; past the caches)
@pytest.mark.parametrize("B,Hkv,nk,keep,room,lens,d", [(2, 2, 300, 100, 130, (300, 7), 64), (3, 1, 90, 120, 120, (90, 0, 1), 128), (2, 2, 300, 100, 3000, (300, 7), 64),
                                                       (3, 2, 5000, 700, 5000, (5000, 0, 333), 128), (2, 2, 777, 300, 777, (5000, 301), 256),
                                                       (2, 4, 30000, 20000, 40000, (30000, 12345), 128)])
@pytest.mark.parametrize("layout", ["HND", "NHD"])
def test_places_behind_what_is_kept(B, Hkv, nk, keep, room, lens, d, layout):
    pa = _pa()
    print(f"evict, zeros behind: B={B} Hkv={Hkv} {nk} -> {keep} of {room}, lens={lens} d={d} {layout}", flush=True)
    k, v, w = _caches(B, Hkv, nk, d, layout, nk)
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    sink, recent = 3, min(40, keep - 3)
    # through the structure, over outputs that hold something
    rows = (B, room, Hkv, d) if layout == "NHD" else (B, Hkv, room, d)
    outs = (torch.full(rows, 5.0, dtype=k.dtype, device="cuda"), torch.full(rows, 6.0, dtype=k.dtype, device="cuda"), torch.full((B, Hkv, room), 7.0, device="cuda"),
            torch.full((B, Hkv, keep), -8, dtype=torch.int32, device="cuda"), torch.full((B,), -9, dtype=torch.int32, device="cuda"))
    a = pa.binding.sage_cache_evict_args()
    a.k, a.v, a.weights, a.kv_lens = k.data_ptr(), v.data_ptr(), w.data_ptr(), lens.data_ptr()
    a.k_out, a.v_out, a.weights_out, a.kept, a.lens_out = (t.data_ptr() for t in outs)
    a.B, a.H_kv, a.N_kv, a.N_keep, a.d, a.sink, a.recent, a.dtype, a.layout, a.N_out = B, Hkv, nk, keep, d, sink, recent, 1, int(layout == "NHD"), room
    a.stream, a.clear = torch.cuda.current_stream().cuda_stream, 1
    assert pa.load_library().sage_cache_evict(ctypes.byref(a)) == 0
    torch.cuda.synchronize()
    _expect(k, v, w, keep, sink, recent, lens, layout, outs)
    # outputs made by the call, of memory that held something
    for t in outs[:4]:
        t.fill_(9)
    del outs
    made = pa.sage_cache_evict(k, v, w, keep, sink=sink, recent=recent, kv_lens=lens, layout=layout, room=room)
    _expect(k, v, w, keep, sink, recent, lens, layout, made)
    # some made, some given: the given ones keep what they hold
    given = torch.full((B, Hkv, room), 7.0, device="cuda")
    ko, vo, wo, kept, left = pa.sage_cache_evict(k, v, w, keep, sink=sink, recent=recent, kv_lens=lens, layout=layout, room=room, weights_out=given)
    for b in range(B):
        n = left[b].item()
        assert (wo[b, :, n:] == 7).all() and (ref.heads_first(ko, layout)[b, :, n:] == 0).all() and (kept[b, :, n:] == 0).all()


def test_replays():
    pa = _pa()
    k, v, w = _caches(2, 2, 3000, 128, "HND", 1)
    lens = torch.tensor([3000, 100], dtype=torch.int32, device="cuda")
    pa.sage_cache_evict(k, v, w, 500, kv_lens=lens, room=3000)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = pa.sage_cache_evict(k, v, w, 500, sink=3, recent=9, kv_lens=lens, room=3000)
    for n in (3000, 400, 0, 2000):
        lens.fill_(n)
        w.copy_(w.flip(-1))
        for t in outs:
            t.fill_(11)
        graph.replay()
        again = pa.sage_cache_evict(k, v, w, 500, sink=3, recent=9, kv_lens=lens, room=3000)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, again)), n


def test_a_bound_above_what_there_is():
    """Up to 4000 tokens of 32 heads under a bound of 16384: all stay, in their order, and zeros behind them."""
    pa = _pa()
    k, v, w = _caches(4, 8, 4000, 128, "HND", 3)
    lens = torch.tensor([4000, 0, 1, 3999], dtype=torch.int32, device="cuda")
    outs = pa.sage_cache_evict(k, v, w, 16384, sink=4, recent=64, kv_lens=lens)
    _expect(k, v, w, 16384, 4, 64, lens, "HND", outs)
