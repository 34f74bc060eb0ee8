"""Norms with rotation of rows from the smallest numbers to the largest: what has to fit FP32 is a row's values, not their squares."""
import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu


def _pa():
    import paper_2411_10958_amd as pa
    pa.load_library()
    return pa


def _rows(shape, exponents, seed):
    """bf16 values, each row times a power of two."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    e = torch.tensor(exponents, device="cuda", dtype=torch.float64)[torch.randint(len(exponents), (*shape[:3], 1), generator=g, device="cuda")]
    x = torch.randn(shape, generator=g, device="cuda").bfloat16().double().clamp(-3.9, 3.9)
    return (x * torch.exp2(e)).bfloat16()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-6, 1e30])
def test_rows_of_any_size(d, eps, interleaved):
    """The bounds of the reference hold over the whole range: scaling a row by a power of two rounds nothing.  Gradients go down with the rows so that theirs, which go with the rows'
    inverse, fit bf16."""
    pa = _pa()
    exponents = [-130, -120, -100, -80, -64, -62, -58, -50, -48, -31, -30, -29, -20, 0, 20, 48, 49, 50, 51, 58, 60, 61, 62, 63, 64, 66, 90, 120, 125]
    for layout, shift in (("HND", 0), ("NHD", 0), ("NHD", 1)):
        B, H, Hkv, N = 2, 5, 2, 33
        q, k = _rows((B, H, N, d), exponents, d), _rows((B, Hkv, N, d), exponents, d + 1)
        f = pa.sage_rope_frequencies(d // 2)
        g = torch.Generator(device="cuda")
        g.manual_seed(d)
        w = [torch.randn(d, generator=g, device="cuda").add_(1.0) for _ in range(2)]
        grads = [(torch.randn(x.shape, generator=g, device="cuda").double() * x.double().square().mean(-1, keepdim=True).sqrt().clamp(2.0 ** -110, 1.0)).bfloat16() for x in (q, k)]
        def put(x):
            x = ref.to_layout(x, layout)
            room = torch.zeros((*x.shape[:3], d + shift), dtype=x.dtype, device="cuda")
            room[..., shift:] = x
            return room[..., shift:]
        q, k, dq_out, dk_out = (put(x) for x in (q, k, *grads))
        pos = torch.arange(N, device="cuda")
        print(f"norm range d={d} eps={eps} {layout} shift={shift}", flush=True)
        y = pa.sage_qk_norm_rope(q, k, f, *w, eps=eps, interleaved=interleaved, layout=layout)
        dx = pa.sage_qk_norm_rope_bwd(dq_out, q, dk_out, k, f, *w, eps=eps, interleaved=interleaved, layout=layout)
        torch.cuda.synchronize()
        eps64 = float(torch.tensor(eps, dtype=torch.float32))
        for i, (name, x, dy) in enumerate((("q", q, dq_out), ("k", k, dk_out))):
            ref.check(name, y[i], *pref.norm_rope(x, w[i], f, pos, eps64, interleaved, 1.0, layout))
            want, bound, want_w, bound_w = pref.norm_rope_bwd(dy, x, w[i], f, pos, eps64, interleaved, 1.0, layout)
            ref.check("d" + name, dx[i], want, bound)
            ref.check(f"d{name}_weight", dx[2 + i], want_w, bound_w)


@pytest.mark.parametrize("value", [3e38, 2e18, 1.9e19, 1e18, 1e-18, 1e-20, 1e-38, 1e-40])
def test_constant_rows(value):
    """A constant row's norm is its sign, without eps."""
    pa = _pa()
    for d in (64, 128, 256):
        q = torch.full((1, 2, 3, d), value, device="cuda").bfloat16()
        q[:, 1] *= -1
        y = pa.sage_qk_norm_rope(q, eps=0.0)
        assert (y[:, 0] == 1).all() and (y[:, 1] == -1).all()
    zero = torch.zeros((1, 1, 1, 64), device="cuda").bfloat16()
    assert pa.sage_qk_norm_rope(zero, eps=0.0).isnan().all() and (pa.sage_qk_norm_rope(zero, eps=1e-38) == 0).all()
