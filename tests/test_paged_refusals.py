"""What the norms with rotation, the append to a cache in pages and its attention refuse, on the host and before anything is launched: no GPU."""
import ctypes
import math
import os

import pytest

P = 1 << 20              # stands for a device pointer: a call that is refused never follows it


def _pa():
    import paper_2411_10958_amd as pa
    if not os.path.exists(pa.lib_path()):
        pytest.skip("libsageattn.so is not built (run __graft_entry__.build())")
    return pa, pa.load_library()


def _status(pa, lib, name, base, **kw):
    a = getattr(pa.binding, name + "_args")()
    for n, x in {**base, **kw}.items():
        if n.endswith("strides"):
            getattr(a, n)[:] = x
        else:
            setattr(a, n, x)
    return getattr(lib, name)(ctypes.byref(a))


# pointers far enough apart for the tensors of the base calls not to overlap
NORM = dict(q=P, k=2 * P, q_out=3 * P, k_out=4 * P, q_weight=5 * P, k_weight=6 * P, B=1, H=2, H_kv=1, N=1, d=64, rot_dim=64, dtype=1, inv_freq=7 * P, eps=1e-6)
BWD = dict(dq_out=8 * P, dk_out=9 * P, q=P, k=2 * P, dq=3 * P, dk=4 * P, q_weight=5 * P, k_weight=6 * P, dq_weight=10 * P, dk_weight=11 * P, B=1, H=2, H_kv=1, N=1, d=64,
           rot_dim=64, dtype=1, inv_freq=7 * P, eps=1e-6, workspace=12 * P, workspace_bytes=1 << 19)

BOTH = [
    (dict(q=0), -1), (dict(k=0), -1), (dict(inv_freq=0), -1), (dict(q=P + 1), -1), (dict(inv_freq=7 * P + 4), -1), (dict(positions=P + 2), -1),
    (dict(positions_stride=-1), -1), (dict(q_weight=5 * P + 2), -1), (dict(q_weight=5 * P + 1, weight_type=1), -1), (dict(B=0), -1), (dict(H=0), -1), (dict(N=-1), -1), (dict(H_kv=0), -1),
    (dict(rot_dim=-2), -1), (dict(rot_dim=3), -2), (dict(rot_dim=66), -2), (dict(d=80), -2), (dict(d=512), -2), (dict(dtype=2), -2), (dict(layout=2), -2), (dict(weight_type=2), -2),
    (dict(interleaved=2), -2), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1), (dict(scale=math.nan), -1), (dict(N=(1 << 24) + 1), -2), (dict(B=65536), -2),
    (dict(offset=(1 << 52) + 1), -1), (dict(q_strides=(-1, 64, 64)), -1), (dict(N=3, q_strides=(1 << 61, 64, 1 << 55)), -1),
]


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(q_out=0), -1), (dict(k_out=0), -1), (dict(k_out=4 * P + 1), -1), (dict(k=0, k_out=0), -1), (dict(N=3, q_out_strides=(384, 64, 64)), -1),
    (dict(N=3, q_out_strides=(384, 0, 128)), -1), (dict(B=2, k_out_strides=(32, 64, 64)), -1),
    (dict(N=3, q_out=P, q_strides=(384, 192, 64), q_out_strides=(384, 64, 128)), -1),       # in place, but rows in another order
    (dict(q_out=2 * P), -1), (dict(k_out=3 * P), -1), (dict(k_out=P), -1), (dict(q_out=5 * P), -1), (dict(k_out=7 * P), -1), (dict(q_out=P + 64), -1),
])
def test_norm(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_qk_norm_rope", NORM, **kw) == status


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(dq=0), -1), (dict(dk=0), -1), (dict(dq_out=0), -1), (dict(dk_out=0), -1), (dict(dq_weight=10 * P + 2), -1), (dict(k=0, dk_out=0, dk=0, k_weight=0), -1),
    (dict(workspace=0), -3), (dict(workspace_bytes=8), -3), (dict(workspace=12 * P + 16), -3), (dict(dq=P), -1), (dict(dk=9 * P + 64), -1), (dict(dq=9 * P), -1),
    (dict(dq_weight=P), -1), (dict(dq_weight=11 * P), -1), (dict(dk_weight=12 * P), -1), (dict(dq_weight=5 * P), -1), (dict(dq=10 * P), -1), (dict(workspace=8 * P), -1),
])
def test_norm_bwd(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_qk_norm_rope_bwd", BWD, **kw) == status


@pytest.mark.parametrize("B,N", [(4, 1 << 24), (16, 1 << 22), (5, 13421772 + 1), (4 * 5, (1 << 24) // 5 + 1)])
def test_norms_of_more_tokens_than_a_launch_counts(B, N):
    """A workgroup of 256 threads takes four tokens at least, and a launch counts its threads in 32 bits: 2^26 - 4 tokens."""
    pa, lib = _pa()
    assert B * N > (1 << 26) - 4
    assert _status(pa, lib, "sage_qk_norm_rope", NORM, B=B, N=N, H=16, q_out=P, k=0, k_out=0, k_weight=0, rot_dim=0, inv_freq=0, q_weight=0) == -2
    assert _status(pa, lib, "sage_qk_norm_rope_bwd", BWD, B=B, N=N) == -2
    a = pa.sage_qk_norm_rope_bwd_args()
    for n, x in {**BWD, "B": 4, "N": (1 << 24) - 1}.items():
        setattr(a, n, x)
    assert pa.sage_qk_norm_rope_bwd_workspace_bytes(a) > 0
    a.N = 1 << 24
    assert pa.sage_qk_norm_rope_bwd_workspace_bytes(a) == 0


def test_norm_bwd_workspace():
    pa, _ = _pa()
    def size(**kw):
        a = pa.sage_qk_norm_rope_bwd_args()
        for n, x in {**BWD, **kw}.items():
            setattr(a, n, x)
        return pa.sage_qk_norm_rope_bwd_workspace_bytes(a)
    assert size() == 3 * 2 * 64 * 4 and size(N=5000) == 512 * 2 * 64 * 4 and size(dq_weight=0, dk_weight=0) == 0 and size(d=65) == 0 and size(dk_weight=0) > 0


APPEND = dict(k=P, v=2 * P, k_cache=3 * P, v_cache=4 * P, k_scale=5 * P, v_scale=6 * P, page_table=7 * P, kv_lens=8 * P, new_lens=9 * P, B=2, H_kv=2, N=3, d=64, n_pages=5, page=64,
              max_pages=2, dtype=1)
CACHE = [
    (dict(k_cache=0), -1), (dict(v_cache=0), -1), (dict(k_scale=0), -1), (dict(v_scale=0), -1), (dict(page_table=0), -1), (dict(k_cache=3 * P + 8), -1), (dict(v_cache=4 * P + 1), -1),
    (dict(page_table=7 * P + 2), -1), (dict(kv_lens=8 * P + 1), -1), (dict(B=0), -1), (dict(H_kv=0), -1), (dict(N=0), -1), (dict(n_pages=0), -1), (dict(page=0), -1), (dict(page=-32), -1),
    (dict(max_pages=0), -1), (dict(d=96), -2), (dict(page=48), -2), (dict(page=16), -2), (dict(max_pages=1 << 19), -2), (dict(n_pages=1 << 30, page=1 << 20, max_pages=1), -2),
    (dict(dtype=2), -2), (dict(layout=2), -2), (dict(N=(1 << 24) + 1), -2), (dict(B=40000, H_kv=2), -2),
]


@pytest.mark.parametrize("kw,status", CACHE + [
    (dict(k=0), -1), (dict(v=0), -1), (dict(k=P + 1), -1), (dict(new_lens=9 * P + 2), -1), (dict(k_strides=(-1, 0, 64)), -1), (dict(v_strides=(1 << 61, 64, 64)), -1),
    (dict(k_cache=P), -1), (dict(v_cache=3 * P), -1), (dict(v_scale=5 * P), -1), (dict(k_scale=3 * P + 16), -1), (dict(v_cache=7 * P), -1), (dict(k_scale=8 * P), -1),
    (dict(k=3 * P), -1),
])
def test_append(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_cache_append", APPEND, **kw) == status


PAGED = dict(q=P, k_cache=3 * P, v_cache=4 * P, k_scale=5 * P, v_scale=6 * P, out=2 * P, page_table=7 * P, kv_lens=8 * P, q_lens=9 * P, lse=10 * P, B=2, H=4, H_kv=2, N=3, d=64,
             n_pages=5, page=64, max_pages=2, causal=1, dtype=1, workspace=11 * P, workspace_bytes=1 << 19)


@pytest.mark.parametrize("kw,status", CACHE + [
    (dict(q=0), -1), (dict(out=0), -1), (dict(q=P + 8), -1), (dict(out=2 * P + 2), -1), (dict(lse=10 * P + 2), -1), (dict(q_lens=9 * P + 1), -1), (dict(H=3), -1), (dict(H=0), -1),
    (dict(causal=2), -1), (dict(clear=4), -1), (dict(sm_scale=math.inf), -1), (dict(sm_scale=math.nan), -1), (dict(window=-1), -1), (dict(sink=-1), -1), (dict(causal=0, window=5), -1), (dict(B=40000, H=2, H_kv=1), -2), (dict(N=1 << 23), -2),
    (dict(out=3 * P), -1), (dict(lse=2 * P), -1), (dict(lse=P), -1), (dict(out=6 * P), -1), (dict(out=P + 16), -1), (dict(lse=9 * P), -1),
    (dict(max_pages=4096, workspace=0), -3), (dict(max_pages=4096, workspace_bytes=64), -3), (dict(max_pages=4096, workspace=11 * P + 16), -3),
])
def test_paged(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_paged", PAGED, **kw) == status
    if status == -2:
        a = pa.sage_attn_paged_args()
        for n, x in {**PAGED, **kw}.items():
            setattr(a, n, x)
        assert pa.sage_attn_paged_workspace_bytes(a) == 0
