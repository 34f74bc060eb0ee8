"""What the operators around attention refuse, on the host and before anything is launched, and the frequencies: no GPU."""
import ctypes
import math
import os

import pytest
import torch

P = 4096                 # stands for a device pointer: a call that is refused never follows it


def _pa():
    import paper_2411_10958_amd as pa
    if not os.path.exists(pa.lib_path()):
        pytest.skip("libsageattn.so is not built (run __graft_entry__.build())")
    return pa, pa.load_library()


def _args(pa, name, **kw):
    a = getattr(pa.binding, name + "_args")()
    for n, x in kw.items():
        if n.endswith("strides"):
            getattr(a, n)[:] = x
        else:
            setattr(a, n, x)
    return a


def _status(pa, lib, name, base, **kw):
    return getattr(lib, name)(ctypes.byref(_args(pa, name, **{**base, **kw})))


# pointers far enough apart for the outputs of the base calls not to overlap
ROPE = dict(q=P, k=2 * P, q_out=3 * P, k_out=4 * P, B=1, H=2, H_kv=1, N=1, d=64, rot_dim=64, dtype=1, inv_freq=P)


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), -1), (dict(q_out=0), -1), (dict(k_out=0), -1), (dict(k=0), -1), (dict(inv_freq=0), -1), (dict(q=P + 1), -1), (dict(k_out=P + 1), -1),
    (dict(inv_freq=P + 4), -1), (dict(positions=P + 2), -1), (dict(positions_stride=-1), -1), (dict(B=0), -1), (dict(H=0), -1), (dict(N=-1), -1), (dict(H_kv=0), -1),
    (dict(rot_dim=0), -1), (dict(rot_dim=-2), -1), (dict(rot_dim=3), -2), (dict(rot_dim=66), -2), (dict(d=80), -2), (dict(d=512), -2), (dict(dtype=2), -2),
    (dict(layout=2), -2), (dict(interleaved=2), -2), (dict(inverse=-1), -2), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1), (dict(N=(1 << 24) + 1), -2),
    (dict(B=65536), -2), (dict(q_strides=(-1, 64, 64)), -1),
    (dict(N=3, q_out_strides=(384, 64, 64)), -1),                    # tokens on top of heads
    (dict(N=3, q_out_strides=(384, 0, 128)), -1), (dict(B=2, k_out_strides=(32, 64, 64)), -1),
    (dict(N=3, q_out=P, q_strides=(384, 192, 64), q_out_strides=(384, 64, 128)), -1),         # in place, but rows in another order
])
def test_rope(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_rope", ROPE, **kw) == status


SHARED = dict(q=P, k_prefix=P, v_prefix=P, k=P, v=P, out=P, B=2, H=4, H_kv=2, N=1, N_prefix=100, N_kv=50, d=128, dtype=1, workspace=P, workspace_bytes=1 << 40)


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), -1), (dict(out=0), -1), (dict(k_prefix=0), -1), (dict(v_prefix=0), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(q=P + 8), -1), (dict(v=P + 2), -1),
    (dict(kv_lens=P + 2), -1), (dict(lse=P + 1), -1), (dict(B=0), -1), (dict(H=3), -1), (dict(H_kv=0), -1), (dict(N=0), -1), (dict(N_prefix=-1), -1), (dict(N_kv=-1), -1),
    (dict(d=96), -2), (dict(dtype=5), -2), (dict(layout=-1), -2), (dict(N=(1 << 24) + 1), -2), (dict(N_prefix=(1 << 24) + 1), -2), (dict(N_kv=(1 << 24) + 1), -2),
    (dict(B=40000, H=2), -2), (dict(N=1 << 24, B=100), -2),
    (dict(workspace=0, N_prefix=5000), -3), (dict(workspace_bytes=16, N_prefix=5000), -3), (dict(workspace=P + 16, N_prefix=5000), -3),
])
def test_shared_prefix(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_shared_prefix", SHARED, **kw) == status
    if status != -3 and not any(n in kw for n in ("q", "out", "k_prefix", "v_prefix", "k", "v", "kv_lens", "lse")):
        assert pa.sage_attn_shared_prefix_workspace_bytes(_args(pa, "sage_attn_shared_prefix", **{**SHARED, **kw})) == 0


def test_shared_prefix_workspace():
    pa, _ = _pa()
    size = lambda **kw: pa.sage_attn_shared_prefix_workspace_bytes(_args(pa, "sage_attn_shared_prefix", **{**SHARED, **kw}))
    long = dict(N_prefix=5000, N_kv=700)
    assert size(**long) % 256 == 0 and size(**long) >= 2 * 2 * 4 * 130 * 4         # a prefix and an own partial result per row at least
    assert size(**{**long, "N_prefix": 0}) > 0 and size(**{**long, "N_kv": 0}) > 0 and size(N_prefix=0) == size() == 0      # (few keys: none)


WEIGHTS = dict(q=P, k=P, lse=P, weights=P, B=2, H=4, H_kv=2, N=1, N_kv=500, d=128, dtype=1)


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), -1), (dict(k=0), -1), (dict(lse=0), -1), (dict(weights=0), -1), (dict(q=P + 8), -1), (dict(k=P + 4), -1), (dict(lse=P + 2), -1), (dict(weights=P + 1), -1),
    (dict(weights_in=P + 3), -1), (dict(kv_lens=P + 1), -1), (dict(B=0), -1), (dict(H=5), -1), (dict(H_kv=-1), -1), (dict(N=0), -1), (dict(N_kv=0), -1), (dict(d=32), -2),
    (dict(dtype=-1), -2), (dict(layout=3), -2), (dict(N=(1 << 24) + 1), -2), (dict(N_kv=(1 << 24) + 1), -2), (dict(B=40000), -2), (dict(N=1 << 24, H=60000, B=1, H_kv=1), -2),
    (dict(N=9000, N_kv=9000), -3), (dict(N=9000, N_kv=9000, workspace=P + 8, workspace_bytes=1 << 40), -3), (dict(N=9000, N_kv=9000, workspace=P, workspace_bytes=64), -3),
])
def test_key_weights(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_key_weights", WEIGHTS, **kw) == status


EVICT = dict(k=1 << 20, v=2 << 20, weights=3 << 20, k_out=4 << 20, v_out=5 << 20, weights_out=6 << 20, kept=7 << 20, lens_out=8 << 20, B=1, H_kv=2, N_kv=100, N_keep=40,
             d=64, sink=4, recent=8, dtype=1)


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), -1), (dict(v=0), -1), (dict(weights=0), -1), (dict(k_out=0), -1), (dict(v_out=0), -1), (dict(kept=0), -1), (dict(lens_out=0), -1), (dict(k=8), -1),
    (dict(v_out=(5 << 20) + 2), -1), (dict(kept=(7 << 20) + 1), -1), (dict(kv_lens=2), -1), (dict(B=0), -1), (dict(H_kv=0), -1), (dict(N_kv=0), -1), (dict(N_keep=0), -1),
    (dict(sink=-1), -1), (dict(recent=-1), -1), (dict(sink=20, recent=21), -1), (dict(sink=1 << 30, recent=1 << 30), -1), (dict(d=100), -2), (dict(dtype=2), -2),
    (dict(layout=2), -2), (dict(N_kv=(1 << 24) + 1), -2), (dict(N_keep=(1 << 24) + 1), -2), (dict(B=65536), -2),
    (dict(k_out=1 << 20), -1), (dict(v_out=(1 << 20) + 16), -1), (dict(weights_out=3 << 20), -1), (dict(kept=6 << 20), -1), (dict(v_out=4 << 20), -1),
])
def test_cache_evict(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_cache_evict", EVICT, **kw) == status


@pytest.mark.parametrize("kw,status", [(dict(N_out=39), -1), (dict(N_out=-1), -1), (dict(N_out=(1 << 24) + 1), -2),
                                       (dict(k_out=(1 << 20) - 2 * 300 * 64 * 2 + 16, N_out=300), -1), (dict(kept=(6 << 20) + 2 * 300 * 4 - 4, N_out=300), -1)])
def test_cache_evict_room(kw, status):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_cache_evict", EVICT, **kw) == status


def test_more_than_a_launch_can_hold():
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_shared_prefix", SHARED, B=1, H=32, H_kv=8, N=(1 << 19) + 1) == -2
    size = lambda n: pa.sage_attn_shared_prefix_workspace_bytes(_args(pa, "sage_attn_shared_prefix", **{**SHARED, **dict(B=1, H=32, H_kv=8, N=n, N_prefix=5000)}))
    assert size((1 << 19) + 1) == 0 and size(1 << 19) > 0
    assert _status(pa, lib, "sage_attn_key_weights", WEIGHTS, B=1, H=8, H_kv=1, N=1 << 24, N_kv=1 << 24) == -2
    assert _status(pa, lib, "sage_attn_key_weights", WEIGHTS, B=8000, H=8, H_kv=8, N=70, N_kv=1 << 24) == -2


def test_null_arguments():
    pa, lib = _pa()
    for name in ("sage_rope", "sage_attn_shared_prefix", "sage_attn_key_weights", "sage_cache_evict"):
        assert getattr(lib, name)(None) == -1
    assert lib.sage_attn_shared_prefix_workspace_bytes(None) == 0 and lib.sage_attn_key_weights_workspace_bytes(None) == 0


def test_the_structures_are_those_of_the_header(tmp_path):
    """Sizes and offsets of every field, by the C compiler."""
    import subprocess
    pa, _ = _pa()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["sage_rope_args", "sage_attn_shared_prefix_args", "sage_attn_key_weights_args", "sage_cache_evict_args"]
    lines = ['#include "sage_attn.h"', "#include <stdio.h>", "int main(void) {"]
    want = []
    for n in names:
        s = getattr(pa.binding, n)
        lines.append(f'printf("%zu\\n", sizeof({n}));')
        want.append(ctypes.sizeof(s))
        for field, _ in s._fields_:
            lines.append(f'printf("%zu\\n", offsetof({n}, {field}));')
            want.append(getattr(s, field).offset)
    src, exe = tmp_path / "t.c", tmp_path / "t"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == want


def test_frequencies():
    pa, lib = _pa()
    f = lambda *a, **kw: pa.sage_rope_frequencies(*a, device="cpu", **kw)
    i = torch.arange(64, dtype=torch.float64)
    plain = 10000.0 ** (-2 * i / 128)
    close = lambda a, b: torch.allclose(a, b, rtol=1e-14, atol=0)        # (64-bit powers: some units of 2^-53)
    assert close(f(128), plain) and f(128).dtype == torch.float64
    assert close(f(128, scaling="linear", factor=4.0), plain / 4)
    base = f(128, scaling="base", factor=4.0)
    assert base[0] == 1 and abs(base[-1] / (plain[-1] / 4) - 1) < 1e-12 and (base[1:] < plain[1:]).all()
    parts = f(128, scaling="parts", factor=8.0, original_length=4096, low=1.0, high=32.0)
    turns = 4096 * plain / (2 * math.pi)
    assert close(parts[turns >= 32], plain[turns >= 32]) and close(parts[turns <= 1], plain[turns <= 1] / 8)
    between = (turns > 1) & (turns < 32)
    share = (turns - 1) / 31
    assert between.any() and close(parts[between], (plain * (share + (1 - share) / 8))[between])
    for kw in (dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=7), dict(base=1.0), dict(base=math.nan), dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=math.inf),
               dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, original_length=100, low=5.0, high=5.0), dict(scaling="base", factor=2.0, rot_dim=2)):
        with pytest.raises(pa.SageError):
            f(**{"rot_dim": 64, **kw})
    with pytest.raises(KeyError):
        f(64, scaling="cubic")
    out = (ctypes.c_double * 4)()
    assert lib.sage_rope_frequencies(8, 10.0, 4, 1.0, 0.0, 0.0, 0.0, out) == -2 and lib.sage_rope_frequencies(8, 10.0, 0, 1.0, 0.0, 0.0, 0.0, None) == -1


def test_tensors_must_be_on_a_gpu():
    pa, _ = _pa()
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    w = torch.zeros((1, 2, 3))
    f = torch.zeros(32, dtype=torch.float64)
    for call in (lambda: pa.sage_rope(x, x, f), lambda: pa.sage_attn_shared_prefix(x, x[0], x[0], x, x), lambda: pa.sage_attn_key_weights(x, x, w),
                 lambda: pa.sage_cache_evict(x, x, w, 2)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pa.sage_cache_evict(x.float(), x, w, 2)
