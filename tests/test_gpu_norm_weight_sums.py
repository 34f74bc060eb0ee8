"""The weights' gradients of the norms against float64, closely enough that no workgroup's sum can be missing."""
import pytest
import torch

import operator_reference as ref
import paged_reference as pref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,Hkv,N,d,dt,layout,rows", [(1, 7, 3, 9000, 128, torch.bfloat16, "NHD", 10), (3, 5, 1, 2500, 256, torch.float16, "HND", 8),
                                                        (2, 9, 2, 3333, 64, torch.bfloat16, "HND", 4), (1, 1, 1, 5000, 128, torch.float16, "NHD", 1), (1, 2, 1, 1, 64, torch.bfloat16, "HND", 2)])
def test_sums_over_rows(B, H, Hkv, N, d, dt, layout, rows):
    """What a sum is off by: 32 units of 2^-24 of each term (the row's root and the rotation), the FP32 sums of the `rows` of q and k that a thread takes at most, the four joins of a
    wavefront and two of a workgroup, and the result's own; sums over workgroups are FP64.  (512 workgroups at most of 256 threads, d / 16 of them a row: 9000 tokens of 10 heads of 128 are 2250 groups of
    4 tokens and 8 heads at a time, five groups to a workgroup and two heads to a thread.)  What one workgroup adds, the root of 1 / 512 of the rows, is tens of times that."""
    import paper_2411_10958_amd as pa
    pa.load_library()
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    make = lambda heads: ref.to_layout(torch.randn((B, heads, N, d), generator=g, device="cuda").to(dt), layout)
    q, k, dq_out, dk_out = make(H), make(Hkv), make(H), make(Hkv)
    w = [torch.randn(d, generator=g, device="cuda").add_(1.0) for _ in range(2)]
    f, pos = pa.sage_rope_frequencies(d), torch.arange(N, device="cuda")
    print(f"weight sums {B}x{H}+{Hkv}x{N}x{d} {dt} {layout}", flush=True)
    got = pa.sage_qk_norm_rope_bwd(dq_out, q, dk_out, k, f, *w, layout=layout)
    torch.cuda.synchronize()
    for name, dw, x, dy, wt, heads in (("q", got[2], q, dq_out, w[0], H), ("k", got[3], k, dk_out, w[1], Hkv)):
        _, _, want, bound = pref.norm_rope_bwd(dy, x, wt, f, pos, 1e-6, False, 1.0, layout)
        terms = (bound - 1e-37) / ((B * heads * N + 32) * ref.F32)
        ref.check(f"d{name}_weight", dw, want, (rows + 7 + 32) * ref.F32 * terms + 1e-37)
