"""Attention over pages in every form that its kernel takes: 16, 32, 64 and 128 rows to a workgroup at every width, with keys in one piece and cut, and with more tiles to a
workgroup than its page numbers are looked up for at a time (16)."""
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


def _workspace(pa, q, c, window=0, sink=0):
    B, H, N, d = q.shape
    pages, Hkv, page, _ = c["k_cache"].shape
    a = pa.sage_attn_paged_args()
    for n, x in dict(B=B, H=H, H_kv=Hkv, N=N, d=d, n_pages=pages, page=page, max_pages=c["page_table"].shape[1], causal=1, window=window, sink=sink,
                     dtype=int(q.dtype == torch.bfloat16)).items():
        setattr(a, n, x)
    return pa.sage_attn_paged_workspace_bytes(a)


def _q(B, H, N, d, dt, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((B, H, N, d), generator=g, device="cuda").to(dt)


def _check(pa, q, c, lens, some=None, **kw):
    """Against the definition, of all sequences or of some; the same without the log-sum-exp."""
    print(f"paged q={tuple(q.shape)} cache={tuple(c['k_cache'].shape)} table={tuple(c['page_table'].shape)} {q.dtype} {kw}", flush=True)
    out, lse = pa.sage_attn_paged(q, **c, kv_lens=lens, return_lse=True, **kw)
    torch.cuda.synchronize()
    some = list(range(len(q))) if some is None else some
    want, wl, ob, lb = pref.paged(q[some], dict(c, page_table=c["page_table"][some]), lens[some], None, True, kw.get("window", 0), kw.get("sink", 0), 0.0, "HND")
    ref.check("lse", lse[some], wl, lb)
    ref.check("out", out[some], want, ob)
    assert torch.equal(pa.sage_attn_paged(q, **c, kv_lens=lens, **kw), out)
    return out


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("N,G", [(4, 4), (5, 4), (8, 4), (9, 4), (12, 4), (13, 3), (16, 4), (33, 1), (8, 8), (17, 4), (33, 4)])
def test_rows_of_a_workgroup(N, G, d, dt):
    """From 16 rows of a KV head to more than 128, 33 to 64 among them, over keys in one piece, in a window with sinks, and in chunks."""
    pa = _pa()
    q = _q(3, 2 * G, N, d, dt, N)
    for cap in (256, 512):
        c = pref.filled(3, 2, cap, 32, d, dt, seed=N)
        assert cap > 256 or _workspace(pa, q, c) == 0
        for lens in ([cap, 77, 3], [cap - 12, 0, 129]):
            _check(pa, q, c, torch.tensor(lens, dtype=torch.int32, device="cuda"))
            _check(pa, q, c, torch.tensor(lens, dtype=torch.int32, device="cuda"), window=60, sink=5)
    c = pref.filled(1, 2, 8192, 64, d, dt, seed=N)
    c["page_table"][0, 7] = -1
    q = _q(1, 2 * G, N, d, dt, N + 1)
    assert _workspace(pa, q, c) > 0
    _check(pa, q, c, torch.tensor([8001], dtype=torch.int32, device="cuda"))
    _check(pa, q, c, torch.tensor([8190], dtype=torch.int32, device="cuda"), window=3000, sink=40)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("N,G", [(1, 4), (5, 4), (12, 4), (40, 4)])
def test_many_tiles_of_a_workgroup_in_every_form(N, G, d, dt):
    """40 tiles, and 34 of a window behind sinks, so that page numbers and scales are looked up again three times: 128 sequences of 4 heads, whose keys are not cut.  (They share the
    pages of three.)"""
    pa = _pa()
    c = pref.filled(3, 4, 5120, 64, d, dt, seed=d)
    c["page_table"][1, 20], c["page_table"][1, 55], c["page_table"][2, 41] = -1, 2 ** 30, -1
    c["page_table"] = c["page_table"][torch.arange(128, device="cuda") % 3].contiguous()
    q = _q(128, 4 * G, N, d, dt, N)
    lens = torch.linspace(5120, 4100, 128).to(torch.int32).cuda()
    some = [0, 1, 2, 70, 127] if N == 1 else [1, 2, 127]
    assert _workspace(pa, q, c) == 0 and _workspace(pa, q, c, 4200, 40) == 0
    _check(pa, q, c, lens, some)
    _check(pa, q, c, lens, some, window=4200, sink=40)


@pytest.mark.parametrize("B,N,G,cap,d", [(64, 12, 4, 8192, 64), (64, 16, 4, 8192, 128), (48, 40, 4, 8192, 256)])
def test_many_tiles_of_a_chunk(B, N, G, cap, d):
    """Two chunks of 32 tiles."""
    pa = _pa()
    c = pref.filled(2, 4, cap, 64, d, torch.bfloat16, seed=d)
    c["page_table"] = c["page_table"][torch.arange(B, device="cuda") % 2].contiguous()
    q = _q(B, 4 * G, N, d, torch.bfloat16, N)
    assert 0 < _workspace(pa, q, c) <= 2 * B * 4 * G * N * (4 * d + 8) + 512
    _check(pa, q, c, torch.linspace(cap, cap - 999, B).to(torch.int32).cuda(), [0, B - 1])
