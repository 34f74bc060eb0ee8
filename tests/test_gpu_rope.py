"""Rotary positions against the rotation in float64: styles, parts of the head, layouts, strides, positions, gradients."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _x(g, B, heads, N, d, dt, layout):
    x = torch.randn((B, heads, N, d), generator=g, device="cuda").mul_(2.0).to(dt)
    return ref.to_layout(x, layout)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 2), (64, 56), (128, 128), (128, 96), (128, 6), (128, 120), (256, 256), (256, 64), (256, 254)])
def test_styles_and_parts_of_the_head(d, rot, interleaved):
    pa = _pa()
    for seed, (B, H, Hkv, N, dt, layout) in enumerate([(1, 1, 1, 1, torch.bfloat16, "HND"), (2, 6, 2, 37, torch.float16, "NHD"), (3, 5, 5, 130, torch.bfloat16, "NHD")]):
        print(f"rope d={d} rot={rot} interleaved={interleaved} B={B} H={H}/{Hkv} N={N} {dt} {layout}", flush=True)
        g = _gen(seed)
        q, k = _x(g, B, H, N, d, dt, layout), _x(g, B, Hkv, N, d, dt, layout)
        f = pa.sage_rope_frequencies(rot)
        pos = torch.randint(-5, 70000, (B, N), generator=g, device="cuda", dtype=torch.int32)
        qo, ko = pa.sage_rope(q, k, f, positions=pos, interleaved=interleaved, scale=1.25, layout=layout)
        for name, x, y in (("q", q, qo), ("k", k, ko)):
            ref.check(name, y, *ref.rope(x, f, pos, interleaved, False, 1.25, layout))
            assert torch.equal(y[..., rot:], x[..., rot:])           # the other channels are copied


@pytest.mark.parametrize("d,rot,interleaved,layout,in_place", [(64, 32, True, "HND", False), (64, 64, True, "NHD", True), (128, 128, False, "NHD", False),
                                                               (256, 128, False, "HND", False), (128, 128, False, "HND", True), (64, 64, False, "HND", False)])
def test_more_than_the_caches_hold(d, rot, interleaved, layout, in_place):
    """Calls that read and write over 256 MB."""
    pa = _pa()
    B, H, Hkv, N = 2, 5, 3, (2 ** 22 // d) + 465
    print(f"rope d={d} rot={rot} interleaved={interleaved} {layout} in place={in_place} N={N}", flush=True)
    g = _gen(d)
    q, k = _x(g, B, H, N, d, torch.bfloat16, layout), _x(g, B, Hkv, N, d, torch.bfloat16, layout)
    f = pa.sage_rope_frequencies(rot)
    pos = torch.arange(N, device="cuda") + 9
    want = [ref.rope(x, f, pos, interleaved, True, 1.0, layout) for x in (q, k)]
    outs = dict(q_out=q, k_out=k) if in_place else {}
    for name, y, (w, bound) in zip("qk", pa.sage_rope(q, k, f, offset=9, interleaved=interleaved, inverse=True, layout=layout, **outs), want):
        ref.check(name, y, w, bound)


def test_more_units_than_a_grid_is_wide():
    """17 million rows at odd addresses: 2^31 threads and more, elements past 2^32."""
    pa = _pa()
    B, N, d = 2, (1 << 23) + 3333, 256
    buf = torch.empty(B * N * (d + 1), dtype=torch.bfloat16, device="cuda")
    for i in range(0, buf.numel(), 1 << 28):
        buf[i:i + (1 << 28)].normal_(generator=_gen(i >> 28))
    q = buf.view(B, 1, N, d + 1)[..., 1:]
    f = pa.sage_rope_frequencies(d)
    y = pa.sage_rope(q, None, f, offset=3)
    for b, n in ((0, 0), (0, N - 500), (1, 0), (1, N // 2), (1, N - 500)):
        pos = torch.arange(n, n + 500, device="cuda") + 3
        ref.check(f"rows {b}, {n}", y[b:b + 1, :, n:n + 500], *ref.rope(q[b:b + 1, :, n:n + 500], f, pos, False, False, 1.0, "HND"))


def test_positions():
    pa = _pa()
    g = _gen(3)
    B, H, N, d = 2, 3, 50, 128
    q = _x(g, B, H, N, d, torch.bfloat16, "HND")
    f = pa.sage_rope_frequencies(d, base=500000.0, scaling="parts", factor=8.0, original_length=8192, low=1.0, high=4.0)
    n = torch.arange(N, device="cuda")
    for kw, pos in ((dict(), n), (dict(offset=2 ** 24 + 7), n + 2 ** 24 + 7), (dict(offset=-1000), n - 1000),
                    (dict(positions=(n * 977).to(torch.int32), offset=5), n * 977 + 5),
                    (dict(positions=torch.full((B, N), 2 ** 31 - 1, dtype=torch.int32, device="cuda")), torch.full((B, N), 2 ** 31 - 1, device="cuda"))):
        y = pa.sage_rope(q, None, f, **kw)
        ref.check(str(list(kw)), y, *ref.rope(q, f, pos, False, False, 1.0, "HND"))


def test_views_of_a_fused_projection_in_place_and_misaligned_rows():
    pa = _pa()
    g = _gen(4)
    B, H, Hkv, N, d = 2, 4, 2, 33, 64
    f = pa.sage_rope_frequencies(d)
    pos = torch.arange(N, device="cuda")
    for pad in (0, 1, 4):                       # rows aligned to 16, 2 and 8 bytes
        row = (H + 2 * Hkv) * d + pad
        print(f"rope of a fused projection, rows of {row} values", flush=True)
        buf = torch.randn((B, N, row), generator=g, device="cuda").to(torch.bfloat16)
        old = buf.clone()
        q, k = (buf[..., a:b].unflatten(-1, (-1, d)) for a, b in ((0, H * d), (H * d, (H + Hkv) * d)))
        qo, ko = pa.sage_rope(q, k, f, layout="NHD")
        assert torch.equal(buf, old) and qo.is_contiguous()
        ref.check("q", qo, *ref.rope(q, f, pos, False, False, 1.0, "NHD"))
        ref.check("k", ko, *ref.rope(k, f, pos, False, False, 1.0, "NHD"))
        pa.sage_rope(q, k, f, layout="NHD", q_out=q, k_out=k)        # in place: the same values, and nothing else
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(buf[..., (H + Hkv) * d:], old[..., (H + Hkv) * d:])
        # into the rows of a cache
        cache = torch.full((B, Hkv, N + 20, d), 7.0, dtype=torch.bfloat16, device="cuda")
        src = old[..., H * d:(H + Hkv) * d].unflatten(-1, (-1, d))
        pa.sage_rope(old[..., :H * d].unflatten(-1, (-1, d)), src, f, layout="NHD", k_out=cache[:, :, 9:9 + N].transpose(1, 2))
        assert torch.equal(cache[:, :, 9:9 + N].transpose(1, 2), ko)
        assert (cache[:, :, :9] == 7).all() and (cache[:, :, 9 + N:] == 7).all()


def test_expanded_inputs_and_strides_that_take_no_step():
    pa = _pa()
    g = _gen(8)
    f = pa.sage_rope_frequencies(64)
    pos = torch.arange(7, device="cuda")
    one = torch.randn((1, 3, 1, 64), generator=g, device="cuda").to(torch.bfloat16)
    x = one.expand(2, 3, 7, 64)                  # the same row at every token
    ref.check("expanded", pa.sage_rope(x, None, f), *ref.rope(x, f, pos, False, False, 1.0, "HND"))
    row = torch.randn(64, generator=g, device="cuda").to(torch.bfloat16)
    with pytest.raises(ValueError):
        pa.sage_rope(row.expand(2, 3, 7, 64), None, f)
    with pytest.raises(pa.SageError):            # an output whose rows share memory
        pa.sage_rope(x.contiguous(), None, f, q_out=x)
    y = torch.randn(2 * 64 * 7 + 1, generator=g, device="cuda").to(torch.bfloat16)
    y = torch.as_strided(y, (1, 2, 7, 64), (3, 448, 64, 1), 0)       # a stride of an extent of one
    ref.check("no step", pa.sage_rope(y, None, f), *ref.rope(y, f, pos, False, False, 1.0, "HND"))


def test_packed_batch_and_channels_that_are_not_turned():
    pa = _pa()
    g = _gen(5)
    x = torch.randn((71, 3, 128), generator=g, device="cuda").to(torch.float16)
    x[5, 1, 100], x[6, 2, 127], x[7, 0, 64] = math.nan, math.inf, -math.inf
    f = pa.sage_rope_frequencies(64)
    pos = torch.cat([torch.arange(40), torch.arange(31)]).to(torch.int32).cuda()
    y = pa.sage_rope(x, None, f, positions=pos)
    want, bound = ref.rope(x[None], f, pos, False, False, 1.0, "NHD")
    ref.check("packed", y[..., :64], want[0, ..., :64], bound[0, ..., :64])
    assert torch.equal(y[..., 64:].contiguous().view(torch.int16), x[..., 64:].contiguous().view(torch.int16))


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(interleaved):
    """The gradient of <w, rope(x)> is the inverse rotation of w: against the formula, and against differences of the float64 form."""
    pa = _pa()
    g = _gen(6)
    f = pa.sage_rope_frequencies(32)
    x, w = (_x(g, 1, 2, 9, 64, torch.float16, "HND") for _ in range(2))
    pos = torch.arange(9, device="cuda") * 331
    got = pa.sage_rope(w, None, f, positions=pos.to(torch.int32), interleaved=interleaved, inverse=True, scale=1.5)
    want, bound = ref.rope(w, f, pos, interleaved, True, 1.5, "HND")
    ref.check("formula", got, want, bound)
    form = lambda t: (ref.rope(t, f, pos, interleaved, False, 1.5, "HND")[0] * w.double()).sum()
    for at in ((0, 0, 3, 1), (0, 1, 8, 20), (0, 0, 5, 40)):
        hi, lo = x.clone(), x.clone()
        hi[at], lo[at] = x[at] + 1.0, x[at] - 1.0
        slope = (form(hi) - form(lo)) / (hi[at].double() - lo[at].double())       # (the rotation is linear: no error but float64's)
        assert abs(got[at].double() - slope) <= bound[at] + 1e-9 * slope.abs()


def test_many_tokens_another_stream_and_replays():
    pa = _pa()
    g = _gen(7)
    f = pa.sage_rope_frequencies(128)
    q, k = _x(g, 2, 8, 3000, 128, torch.bfloat16, "HND"), _x(g, 2, 2, 3000, 128, torch.bfloat16, "HND")
    pos = torch.arange(3000, dtype=torch.int32, device="cuda")
    want = pa.sage_rope(q, k, f, positions=pos)
    ref.check("q", want[0], *ref.rope(q, f, pos, False, False, 1.0, "HND"))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = pa.sage_rope(q, k, f, positions=pos, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.sage_rope(q, k, f, positions=pos, q_out=qo, k_out=ko)
    for step in range(3):
        pos.add_(17)
        graph.replay()
        want = pa.sage_rope(q, k, f, positions=pos)
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1]), step
