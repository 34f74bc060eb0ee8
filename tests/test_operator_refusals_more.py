"""More of what the operators around attention refuse on the host, before anything is launched: no GPU."""

import pytest

from test_operator_refusals import EVICT, _pa, _status


@pytest.mark.parametrize("clear", [2, -1, 256])
def test_cache_evict_clear(clear):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_cache_evict", EVICT, clear=clear) == -2


D = 64
BIG = 1 << 40            # (addresses nothing is at)


def _meet(x, sx, ex, y, sy, ey):
    """Whether two sets of rows of D values share one, value by value."""
    rows = lambda at, s, e: {at // 2 + s[0] * b + s[1] * h + s[2] * n for b in range(e[0]) for h in range(e[1]) for n in range(e[2])}
    return any(abs(i - j) < D for i in rows(x, sx, ex) for j in rows(y, sy, ey))


def _rope_overlap(q, qs, k, ks, qo, qos, ko, kos, B, H, Hkv, N):
    """What the call should say of these tensors: True if it has to refuse them."""
    tensors = [(q, qs, (B, H, N)), (k, ks, (B, Hkv, N)), (qo, qos, (B, H, N)), (ko, kos, (B, Hkv, N))]
    for y in (2, 3):
        for x in range(y):
            if not (x == y - 2 and tensors[x][0] == tensors[y][0]) and _meet(*tensors[x], *tensors[y]):
                return True
    return False


def test_rope_refuses_outputs_that_overlap_another_tensor():
    """Outputs that would be written while they are read, or twice; what is right (the last of the cases) is not called here."""
    pa, lib = _pa()
    B, H, Hkv, N = 2, 4, 2, 3
    row = (H + 2 * Hkv) * D
    fused = (N * row, D, row)                                            # slices of a fused projection, token-major
    heads = lambda h: (h * N * D, N * D, D)
    base = dict(B=B, H=H, H_kv=Hkv, N=N, d=D, rot_dim=D, dtype=1, inv_freq=1 << 20, layout=1)
    far = BIG + (1 << 30)
    cases = [
        (BIG + 2 * row, fused),                                          # q_out: q a token later
        (BIG + 2 * D, fused),                                            # .. a head later
        (BIG + 2 * H * D, fused),                                        # .. where k is
        (BIG + 2 * (H * D - 1), fused),                                  # .. one value before k
        (BIG + 2, heads(H)),                                             # head-major over token-major
        (BIG + 2 * (B * N * row - D), heads(H)),                         # .. its first row over the last of the projection, which is neither q nor k
    ]
    seen = []
    for qo, qos in cases:
        x = (BIG, fused, BIG + 2 * H * D, fused, qo, qos, far, heads(Hkv), B, H, Hkv, N)
        seen.append(_rope_overlap(*x))
        if seen[-1]:
            assert _status(pa, lib, "sage_rope", base, q=BIG, q_strides=fused, k=BIG + 2 * H * D, k_strides=fused, q_out=qo, q_out_strides=qos, k_out=far,
                           k_out_strides=heads(Hkv)) == -1, (qo, qos)
    assert seen == [True, True, True, True, True, False]
    # outputs over each other, and each over the other's input
    for kw in (dict(q_out=far, k_out=far + 2 * 5 * D), dict(q_out=far, k_out=BIG), dict(q_out=BIG + 2 * H * D, k_out=far)):
        assert _status(pa, lib, "sage_rope", base, q=BIG, q_strides=fused, k=BIG + 2 * H * D, k_strides=fused, q_out_strides=heads(H), k_out_strides=heads(Hkv), **kw) == -1


def test_rope_refuses_strides_past_any_memory():
    pa, lib = _pa()
    base = dict(q=BIG, q_out=BIG << 1, H=2, N=3, B=2, d=D, rot_dim=D, dtype=1, inv_freq=1 << 20)
    for kw in (dict(q_strides=((1 << 62), D, 2 * D)), dict(q_out_strides=((1 << 62), D, 2 * D)), dict(q_strides=(1 << 10, D, 1 << 50))):
        assert _status(pa, lib, "sage_rope", base, **kw) == -1


KW = dict(q=1 << 20, k=2 << 20, lse=3 << 20, weights_in=4 << 20, weights=5 << 20, kv_lens=6 << 20, B=2, H=4, H_kv=2, N=1, N_kv=500, d=128, dtype=1)


@pytest.mark.parametrize("kw", [dict(weights=(4 << 20) + 4), dict(weights=(4 << 20) - 4), dict(weights=(4 << 20) + 2 * 2 * 500 * 4 - 4), dict(weights=1 << 20), dict(weights=(2 << 20) + 16),
                                dict(weights=3 << 20), dict(weights=(6 << 20) + 4), dict(weights=(6 << 20) - 2 * 2 * 500 * 4 + 4)])
def test_key_weights_overlaps(kw):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_key_weights", KW, **kw) == -1


@pytest.mark.parametrize("at", [1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20])
def test_key_weights_workspace_over_a_tensor(at):
    pa, lib = _pa()
    far = dict(q=1 << 30, k=2 << 30, lse=3 << 30, weights_in=4 << 30, weights=5 << 30, kv_lens=6 << 30)
    assert _status(pa, lib, "sage_attn_key_weights", {**KW, **far}, N=9000, N_kv=9000, workspace=at << 10, workspace_bytes=1 << 40) == -1


SP = dict(q=1 << 30, k_prefix=2 << 30, v_prefix=3 << 30, k=4 << 30, v=5 << 30, out=6 << 30, lse=7 << 30, kv_lens=8 << 30, B=2, H=4, H_kv=2, N=1, N_prefix=5000, N_kv=700, d=128, dtype=1,
          workspace=9 << 30, workspace_bytes=1 << 29)


@pytest.mark.parametrize("kw", [dict(out=(1 << 30) + 256), dict(out=2 << 30), dict(out=(3 << 30) + 2 * 5000 * 256 - 16), dict(out=4 << 30), dict(out=(5 << 30) - 16), dict(out=(7 << 30) + 16),
                                dict(out=8 << 30), dict(lse=1 << 30), dict(lse=(2 << 30) + 4), dict(lse=8 << 30), dict(lse=(9 << 30) + 256), dict(workspace=1 << 30), dict(workspace=4 << 30),
                                dict(workspace=6 << 30), dict(workspace=(5 << 30) + 256)])
def test_shared_prefix_overlaps(kw):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_attn_shared_prefix", SP, **kw) == -1


def test_workspaces_are_sized_with_public_names():
    pa, _ = _pa()
    a = pa.sage_attn_shared_prefix_args(B=2, H=4, H_kv=2, N=1, N_prefix=5000, N_kv=700, d=128, causal=1, dtype=pa.SAGE_DT_BF16)
    assert pa.sage_attn_shared_prefix_workspace_bytes(a) > 0
    a = pa.sage_attn_key_weights_args(B=1, H=4, H_kv=1, N=3001, N_kv=3001, d=64, causal=1, dtype=pa.SAGE_DT_FP16, layout=1)
    assert pa.sage_attn_key_weights_workspace_bytes(a) > 0
    assert {"sage_attn_shared_prefix_args", "sage_attn_key_weights_args"} <= set(pa.__all__)


@pytest.mark.parametrize("kw", [dict(N_prefix=131072, N_kv=512), dict(N_prefix=0, N_kv=131072), dict(N_prefix=131072, N_kv=0)])
def test_long_keys_of_one_head_are_cut_for_the_whole_chip(kw):
    """A call bound by reading, with one KV head: as many partial results as a row may have, 256, which the workspace has room for."""
    pa, _ = _pa()
    a = pa.sage_attn_shared_prefix_args(B=1, H=8, H_kv=1, N=1, d=128, causal=1, dtype=pa.SAGE_DT_BF16, **kw)
    assert pa.sage_attn_shared_prefix_workspace_bytes(a) == 256 * 8 * (128 + 2) * 4


def test_frequencies_of_a_base_raised_past_64_bits():
    pa, _ = _pa()
    for rot, base, factor in ((64, 1e300, 1e10), (4, 10000.0, 1e200)):
        with pytest.raises(pa.SageError):
            pa.sage_rope_frequencies(rot, base=base, scaling="base", factor=factor, device="cpu")
    assert pa.sage_rope_frequencies(64, base=1e300, scaling="base", factor=2.0, device="cpu")[-1] > 0


@pytest.mark.parametrize("offset", [(1 << 52) + 1, -(1 << 52) - 1, (1 << 63) - 1, -(1 << 63)])
def test_rope_offsets_that_are_no_whole_numbers_in_64_bits(offset):
    pa, lib = _pa()
    assert _status(pa, lib, "sage_rope", dict(q=BIG, q_out=BIG << 1, H=2, N=3, B=2, d=D, rot_dim=D, dtype=1, inv_freq=1 << 20), offset=offset) == -1
