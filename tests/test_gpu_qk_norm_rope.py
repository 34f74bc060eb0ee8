"""Norms of queries and keys with their rotation, and the gradient, against float64."""
import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _gen(seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(B, H, Hkv, N, d, dt, layout, fused=False, seed=0, std=3.0):
    """q, k (views of one buffer if fused, with room behind the keys), weights."""
    g = _gen(seed)
    def two(std):
        if fused:
            x = torch.randn((B, N, H + 2 * Hkv, d), generator=g, device="cuda").mul_(std).to(dt)
            q, k = x[:, :, :H], x[:, :, H:H + Hkv]
            return (q, k) if layout == "NHD" else (q.transpose(1, 2), k.transpose(1, 2))
        return tuple(ref.to_layout(torch.randn((B, h, N, d), generator=g, device="cuda").mul_(std).to(dt), layout) for h in (H, Hkv))
    q, k = two(std)
    dq, dk = two(1.0)
    w = [torch.randn(d, generator=g, device="cuda").add_(1.0) for _ in range(2)]
    return q, k, dq, dk, w


def _check(pa, x, f, positions, weights=True, same=False, eps=1e-6, interleaved=False, scale=1.0, layout="HND", **kw):
    q, k, dq_out, dk_out, w = x
    print(f"norm q={tuple(q.shape)} k={tuple(k.shape)} {q.dtype} {layout} rot={0 if f is None else 2 * len(f)} interleaved={interleaved}", flush=True)
    w = [(y.to(q.dtype) if same else y) if weights else None for y in w]
    common = dict(q_weight=w[0], k_weight=w[1], eps=eps, positions=positions, interleaved=interleaved, scale=scale, layout=layout)
    yq, yk = pa.sage_qk_norm_rope(q, k, f, **common, **kw)
    dq, dk, dqw, dkw = pa.sage_qk_norm_rope_bwd(dq_out, q, dk_out, k, f, **common)
    torch.cuda.synchronize()
    N = q.shape[1] if layout == "NHD" else q.shape[2]
    pos = positions if positions is not None else torch.arange(N, device="cuda")
    for name, y, dx, dw, src, dy, wt in (("q", yq, dq, dqw, q, dq_out, w[0]), ("k", yk, dk, dkw, k, dk_out, w[1])):
        ref.check(name, y, *pref.norm_rope(src, wt, f, pos, eps, interleaved, scale, layout))
        want, bound, want_w, bound_w = pref.norm_rope_bwd(dy, src, wt, f, pos, eps, interleaved, scale, layout)
        ref.check("d" + name, dx, want, bound)
        if weights:
            ref.check(f"d{name}_weight", dw, want_w, bound_w)
        else:
            assert dw is None
    return yq, yk, dq, dk, dqw, dkw


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,Hkv,N", [(1, 1, 1, 1), (2, 4, 2, 1), (3, 5, 1, 7), (2, 8, 8, 33), (1, 6, 2, 260), (2, 32, 8, 129)])
def test_sizes(B, H, Hkv, N, d):
    pa = _pa()
    dt, layout = (torch.bfloat16, "HND") if (B + N + d // 64) % 2 else (torch.float16, "NHD")
    pos = torch.randint(0, 100000, (B, N), generator=_gen(1), device="cuda").to(torch.int32)
    _check(pa, _inputs(B, H, Hkv, N, d, dt, layout), pa.sage_rope_frequencies(d, base=500000.0), pos, layout=layout, same=N % 2 == 0)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 2), (64, 24), (128, 64), (128, 120), (128, 32), (256, 6), (256, 128), (256, 250)])
def test_partial_rotations(d, rot, interleaved):
    pa = _pa()
    for layout, fused in (("HND", False), ("NHD", True)):
        _check(pa, _inputs(2, 4, 2, 19, d, torch.bfloat16, layout, fused=fused), pa.sage_rope_frequencies(rot), None, interleaved=interleaved, layout=layout, scale=1.25)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_no_rotation_and_no_weights(d):
    pa = _pa()
    x = _inputs(2, 4, 2, 19, d, torch.float16, "HND")
    _check(pa, x, None, None)
    _check(pa, x, None, None, weights=False)
    _check(pa, x, pa.sage_rope_frequencies(d), None, weights=False, eps=0.0)
    f = pa.sage_rope_frequencies(d)
    only = pa.sage_qk_norm_rope(x[0], None, f, q_weight=x[4][0])
    both = pa.sage_qk_norm_rope(x[0], x[1], f, q_weight=x[4][0])
    assert torch.equal(only, both[0])
    ref.check("k without a weight", both[1], *pref.norm_rope(x[1], None, f, torch.arange(19, device="cuda"), 1e-6, False, 1.0, "HND"))
    a, b = pa.sage_qk_norm_rope_bwd(x[2], x[0], None, None, f, q_weight=x[4][0]), pa.sage_qk_norm_rope_bwd(x[2], x[0], x[3], x[1], f, k_weight=x[4][1])
    assert a[1] is None and a[3] is None and b[2] is None
    want = pref.norm_rope_bwd(x[2], x[0], x[4][0], f, torch.arange(19, device="cuda"), 1e-6, False, 1.0, "HND")
    ref.check("dq_weight alone", a[2], want[2], want[3])
    want = pref.norm_rope_bwd(x[3], x[1], x[4][1], f, torch.arange(19, device="cuda"), 1e-6, False, 1.0, "HND")
    ref.check("dk_weight alone", b[3], want[2], want[3])


@pytest.mark.parametrize("shift", [1, 4, 8])
def test_views_in_any_order_and_at_any_alignment(shift):
    """Rows that start at odd elements, heads and tokens with room between them, an expanded gradient, outputs in strided views."""
    pa = _pa()
    B, H, Hkv, N, d = 2, 4, 2, 9, 128
    g = _gen(3)
    f = pa.sage_rope_frequencies(96)
    big = torch.randn((B, N, H + Hkv, d + shift), generator=g, device="cuda").mul_(2.0).bfloat16()
    q, k = big[:, :, :H, shift:], big[:, :, H:, shift:]
    dy = torch.randn((1, 1, 1, d), generator=g, device="cuda").bfloat16().expand(B, N, H, d)[:, :, :, :]
    dyk = torch.randn((B, 1, Hkv, d), generator=g, device="cuda").bfloat16().expand(B, N, Hkv, d)
    w = [torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    room = torch.full((B, N, H + Hkv, d + shift), 7.0, device="cuda").bfloat16()
    yq, yk = pa.sage_qk_norm_rope(q, k, f, *w, layout="NHD", q_out=room[:, :, :H, shift:], k_out=room[:, :, H:, shift:])
    pos = torch.arange(N, device="cuda")
    ref.check("q", yq, *pref.norm_rope(q, w[0], f, pos, 1e-6, False, 1.0, "NHD"))
    ref.check("k", yk, *pref.norm_rope(k, w[1], f, pos, 1e-6, False, 1.0, "NHD"))
    assert (room[..., :shift] == 7.0).all()
    with pytest.raises(ValueError, match="expanded"):
        pa.sage_qk_norm_rope_bwd(dy, q, dyk, k, f, *w, layout="NHD")
    dy = torch.randn((B, 1, H, d), generator=g, device="cuda").bfloat16().expand(B, N, H, d)
    room = torch.full((B, N, H + Hkv, d + shift), 7.0, device="cuda").bfloat16()
    dq, dk, dqw, dkw = pa.sage_qk_norm_rope_bwd(dy, q, dyk, k, f, *w, layout="NHD", dq=room[:, :, :H, shift:], dk=room[:, :, H:, shift:])
    for name, dx, dw, src, gy, wt in (("q", dq, dqw, q, dy, w[0]), ("k", dk, dkw, k, dyk, w[1])):
        want, bound, want_w, bound_w = pref.norm_rope_bwd(gy, src, wt, f, pos, 1e-6, False, 1.0, "NHD")
        ref.check("d" + name, dx, want, bound)
        ref.check(f"d{name}_weight", dw, want_w, bound_w)
    assert (room[..., :shift] == 7.0).all()


def test_in_place_and_packed():
    pa = _pa()
    q, k, dq, dk, w = _inputs(1, 4, 2, 50, 64, torch.bfloat16, "NHD")
    f = pa.sage_rope_frequencies(64)
    pos = torch.randint(0, 500, (50,), generator=_gen(1), device="cuda").to(torch.int32)
    want = _check(pa, (q, k, dq, dk, w), f, pos, layout="NHD")
    got = pa.sage_qk_norm_rope(q[0], k[0], f, *w, positions=pos)
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[1][0])
    grads = pa.sage_qk_norm_rope_bwd(dq[0], q[0], dk[0], k[0], f, *w, positions=pos, dq=dq[0], dk=dk[0])
    for a, b in zip(grads, (want[2][0], want[3][0], want[4], want[5])):
        assert torch.equal(a, b)
    pa.sage_qk_norm_rope(q, k, f, *w, positions=pos, layout="NHD", q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_the_gradient_against_differences(dt):
    """Along a direction, the differences of the result in float64 against the kernel's gradient: h^2 of the third derivative and rounding stay below
    10^-6 of the terms."""
    pa = _pa()
    q, k, dq_out, dk_out, w = _inputs(2, 3, 3, 11, 64, dt, "HND", std=1.0)
    f, pos = pa.sage_rope_frequencies(48), torch.arange(11, device="cuda")
    dq, _, dqw, _ = pa.sage_qk_norm_rope_bwd(dq_out, q, dk_out, k, f, *w, interleaved=True)
    g = _gen(9)
    dirx, dirw = torch.randn(q.shape, generator=g, device="cuda", dtype=torch.float64), torch.randn(64, generator=g, device="cuda", dtype=torch.float64)
    def value(t):
        x, wt = q.double() + t * dirx, w[0].double() + t * dirw
        y = x * wt / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        return (pref._turn(y, pref._angle(f, pos), True, 1.0)[0] * dq_out.double()).sum().item()
    h = 1e-5
    slope = (value(h) - value(-h)) / (2 * h)
    _, bound, _, bound_w = pref.norm_rope_bwd(dq_out, q, w[0], f, pos, 1e-6, True, 1.0, "HND")
    terms = (dq.double() * dirx).abs().sum().item() + (dqw.double() * dirw).abs().sum().item()
    room = (bound * dirx.abs()).sum().item() + (bound_w * dirw.abs()).sum().item() + 1e-6 * terms
    assert abs(slope - (dq.double() * dirx).sum().item() - (dqw.double() * dirw).sum().item()) <= room


def test_many_rows():
    """More than the gradient's workgroups take at once, and heads that do not divide."""
    pa = _pa()
    _check(pa, _inputs(1, 7, 3, 9000, 128, torch.bfloat16, "NHD", fused=True), pa.sage_rope_frequencies(128), None, layout="NHD")
    _check(pa, _inputs(3, 5, 1, 2500, 256, torch.float16, "HND"), pa.sage_rope_frequencies(256), None)


def test_values_that_are_not_finite_stay_in_their_row():
    pa = _pa()
    q, k, dq, dk, w = _inputs(2, 3, 2, 9, 128, torch.bfloat16, "HND")
    f = pa.sage_rope_frequencies(128)
    clean, grads = pa.sage_qk_norm_rope(q, k, f, *w), pa.sage_qk_norm_rope_bwd(dq, q, dk, k, f, *w)
    q[0, 1, 4, 7], k[1, 0, 8, 100] = float("nan"), float("inf")
    got, after = pa.sage_qk_norm_rope(q, k, f, *w), pa.sage_qk_norm_rope_bwd(dq, q, dk, k, f, *w)
    for y, z in ((got, clean), (after[:2], grads[:2])):
        assert y[0][0, 1, 4].isnan().all() and y[1][1, 0, 8].isnan().any()
        for a, b, at in ((y[0], z[0], (0, 1, 4)), (y[1], z[1], (1, 0, 8))):
            rest = torch.ones(a.shape[:3], dtype=torch.bool, device="cuda")
            rest[at] = False
            assert torch.equal(a[rest], b[rest])
    zero = pa.sage_qk_norm_rope(torch.zeros_like(q), None, f, w[0])
    assert (zero == 0).all()


def test_the_same_twice_and_on_a_stream():
    pa = _pa()
    x = _inputs(2, 8, 2, 700, 128, torch.bfloat16, "NHD", fused=True)
    f = pa.sage_rope_frequencies(128)
    run = lambda **kw: pa.sage_qk_norm_rope_bwd(x[2], x[0], x[3], x[1], f, *x[4], layout="NHD", **kw)
    want = run()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = run(stream=other)
    torch.cuda.current_stream().wait_stream(other)
    again = run()
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_captured():
    """Forward and backward in one graph, replayed with other inputs and eager work between."""
    pa = _pa()
    f = pa.sage_rope_frequencies(64)
    q, k, dq, dk, w = _inputs(2, 4, 2, 37, 64, torch.bfloat16, "HND")
    keep = [torch.empty_like(t) for t in (q, k, q, k)] + [torch.empty(64, device="cuda") for _ in range(2)]
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    def step():
        pa.sage_qk_norm_rope(q, k, f, *w, q_out=keep[0], k_out=keep[1])
        pa.sage_qk_norm_rope_bwd(dq, q, dk, k, f, *w, dq=keep[2], dk=keep[3], dq_weight=keep[4], dk_weight=keep[5], workspace=room)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        q.copy_(torch.randn(q.shape, generator=_gen(20 + i), device="cuda"))
        w[0].add_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in keep]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, keep):
            assert torch.equal(a, b)
