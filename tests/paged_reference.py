"""Norms with rotation, the cache in 8 bits and pages and its attention in float64, from their definitions, and how far a kernel may be from them.

HALF, TINY and F32 are the half steps of operator_reference.py; the bounds beside the results add up such roundings in the worst case."""
import math

import torch

from operator_reference import F32, HALF, TINY, heads_first

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# ---- norm and rotation --------------------------------------------------------------------------------------------

def _turn(x, angle, interleaved, scale, back=False):
    """x [B, heads, N, d] turned by angle [B, 1, N, rot / 2]; beside it |a| + |b| of each value's pair (times |scale|)."""
    r = 2 * angle.shape[-1]
    c, s = angle.cos() * scale, angle.sin() * scale * (-1 if back else 1)
    ia = torch.arange(0, r, 2) if interleaved else torch.arange(r // 2)
    ib = ia + (1 if interleaved else r // 2)
    y, size = x.clone(), x.abs()
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * abs(scale)
    return y, size


def _angle(f, positions):
    p = positions.double()
    p = p[None, :] if p.dim() == 1 else p
    return p[:, None, :, None] * f.double()


def _normed(x, w, eps, d):
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return r, (torch.ones(d, dtype=torch.float64, device=x.device) if w is None else w.double())


def norm_rope(x, w, f, positions, eps, interleaved, scale, layout):
    """The result and its bound: half a step of the output; the sum of d squares (16 in a thread, 4 joins, the mean, eps: 22 roundings, half of that in r),
    the root (4), two products, and the 8 of a rotation: less than 32 units of 2^-24 of |a| + |b|."""
    dt = x.dtype
    x = heads_first(x, layout).double()
    r, w = _normed(x, w, eps, x.shape[-1])
    n = x * r * w
    y, size = _turn(n, _angle(f, positions), interleaved, scale) if f is not None else (n, n.abs())
    bound = HALF[dt] * y.abs() + TINY[dt] + 32 * F32 * size
    return heads_first(y, layout), heads_first(bound, layout)


def norm_rope_bwd(dy, x, w, f, positions, eps, interleaved, scale, layout):
    """dx, dw and their bounds.  g has the 8 roundings of a rotation; the mean of g w x those, two products and the sum's 22, times r^2 (30 more): less
    than 64 units of what its terms add up to, as is r (g w) with 15 + 8 + 2.  A row's g x r is off by less than 32 units, a sum over R rows by R more."""
    dt = x.dtype
    x, dy = heads_first(x, layout).double(), heads_first(dy, layout).double()
    d = x.shape[-1]
    r, w = _normed(x, w, eps, d)
    g, size = _turn(dy, _angle(f, positions), interleaved, scale, back=True) if f is not None else (dy, dy.abs())
    m = (g * w * x).mean(-1, keepdim=True) * r * r
    dx = r * (g * w - x * m)
    of_m = (size * w.abs() * x.abs()).mean(-1, keepdim=True) * r * r
    bound = HALF[dt] * dx.abs() + TINY[dt] + 64 * F32 * r * (size * w.abs() + x.abs() * of_m)
    terms = (size * x.abs() * r).flatten(0, 2)
    dw = (g * x * r).flatten(0, 2).sum(0)
    return heads_first(dx, layout), heads_first(bound, layout), dw, (len(terms) + 32) * F32 * terms.sum(0) + 1e-37


# ---- the cache ----------------------------------------------------------------------------------------------------

def new_cache(pages, Hkv, page, d, fill=0x7f):
    """(k_cache, v_cache, k_scale, v_scale) full of NaN, as memory that was never written may be."""
    codes = [torch.full((pages, Hkv, page, d), fill, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
    scales = [torch.full((pages, Hkv, page // 32), 0xff, dtype=torch.uint8, device="cuda").view(E8M0) for _ in range(2)]
    return codes + scales


def table(B, cap, page, pages, seed=0):
    """A page table of `cap` tokens a sequence over a pool, in no order."""
    g = torch.Generator().manual_seed(seed)
    n = cap // page
    return torch.randperm(pages, generator=g)[:B * n].reshape(B, n).to(torch.int32).cuda()


def _two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def round_e4m3(y):
    """To the nearest of E4M3's numbers, ties to the even one, cut to 448; NaN stays."""
    _, e = torch.frexp(y)
    step = _two((e - 4).clamp(min=-9))
    return ((y / step).round() * step).clamp(-448, 448)


def append(x, codes, scale, tbl, lens, news, layout):
    """(codes, scales) after the append, float64 on the CPU, token by token of the definition."""
    most = 7 if x.dtype == torch.float16 else 119
    x = heads_first(x, layout).double().cpu()
    codes, scale, tbl = codes.double().cpu(), scale.double().cpu(), tbl.cpu()
    B, Hkv, N, d = x.shape
    pages, _, page, _ = codes.shape
    cap = tbl.shape[1] * page
    for b in range(B):
        n = cap if lens is None else min(max(int(lens[b]), 0), cap)
        count = N if news is None else min(max(int(news[b]), 0), N)
        first = n - count
        start = max(first, 0)
        for t0 in range(start // 32 * 32, n, 32):
            at, j = int(tbl[b, t0 // page]), t0 % page // 32
            lo, hi = max(t0, start), min(t0 + 32, n)
            if hi <= lo or not 0 <= at < pages:
                continue
            new = x[b, :, lo - first:hi - first]
            size = torch.where(new.isfinite(), new.abs(), 0.0).amax((1, 2))
            f, e = torch.frexp(size)
            two = _two(torch.where(size == 0, -64, e - 9 + (f > 0.875).int()).clamp(-64, most))      # (any power of two will do for zeros)
            block = codes[at, :, 32 * j:32 * j + 32]
            if lo > t0:
                two = torch.maximum(two, scale[at, :, j])
                block[:, :lo - t0] = round_e4m3(block[:, :lo - t0] * (scale[at, :, j] / two)[:, None, None])
            y = new / two[:, None, None]
            block[:, lo - t0:hi - t0] = round_e4m3(torch.where(new.isfinite(), y, math.nan))
            scale[at, :, j] = two
    return codes, scale


def same(name, got, want):
    got = got.double().cpu()
    assert got.shape == want.shape
    assert torch.equal(got.nan_to_num(nan=1e300), want.nan_to_num(nan=1e300)), f"{name}: {(got.nan_to_num(nan=1e300) != want.nan_to_num(nan=1e300)).sum().item()} differ"


def filled(B, Hkv, cap, page, d, dt, spare=3, seed=0, spread=1.0):
    """A cache whose every token holds a code, made by the definition, with its table: a dict.  Scales of blocks differ."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pages = B * (cap // page) + spare
    c = dict(page_table=table(B, cap, page, pages, seed))
    for n in "kv":
        x = torch.randn((pages, Hkv, page // 32, 32, d), generator=g, device="cuda", dtype=torch.float64) * spread
        x *= torch.exp2(torch.randint(-3, 4, (pages, Hkv, page // 32, 1, 1), generator=g, device="cuda").double())
        f, e = torch.frexp(x.abs().amax((-1, -2)))
        e = (e - 9 + (f > 0.875).int()).clamp(-64, 7)
        c[n + "_cache"] = round_e4m3(x / _two(e)[..., None, None]).float().to(E4M3).reshape(pages, Hkv, page, d)
        c[n + "_scale"] = (e + 127).to(torch.uint8).view(E8M0)
    return c


def values(c, n, b, h, length):
    """[length, d] values of a sequence and head in float64, and which of its tokens are in a page of the pool."""
    codes, scale, tbl = c[n + "_cache"], c[n + "_scale"], c["page_table"]
    pages, _, page, d = codes.shape
    t = torch.arange(length, device=codes.device)
    at = tbl[b].long()[t // page]
    there = (at >= 0) & (at < pages)
    at = at.clamp(0, pages - 1)
    x = codes.view(torch.uint8)[at, h, t % page].view(E4M3).double() * scale.view(torch.uint8)[at, h, t % page // 32].view(E8M0).double()[:, None]
    return x, there


def paged(q, c, lens, q_lens, causal, window, sink, sm_scale, layout, out_was=None, lse_was=None):
    """out, lse in float64 and their bounds; what is not there keeps out_was and lse_was (None: zeros).  The bounds are those of the 16-bit attention in
    operator_reference.py: codes are exact in the products, and half of fp16's smallest step for a value of V that is below its normal numbers."""
    dt, dev = q.dtype, q.device
    q = heads_first(q, layout).double()
    B, H, N, d = q.shape
    page = c["k_cache"].shape[2]
    cap, Hkv = c["page_table"].shape[1] * page, c["k_cache"].shape[1]
    scale = sm_scale if sm_scale > 0 else 1 / math.sqrt(d)
    out = torch.zeros_like(q) if out_was is None else heads_first(out_was, layout).double().clone()
    lse = torch.zeros((B, H, N), dtype=torch.float64, device=dev) if lse_was is None else lse_was.double().clone()
    ob, lb = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n = cap if lens is None else min(max(int(lens[b]), 0), cap)
        count = N if q_lens is None else min(max(int(q_lens[b]), 0), N)
        if count == 0:
            continue
        t, p = torch.arange(n, device=dev), max(n - count, 0) + torch.arange(count, device=dev)[:, None]
        see = torch.ones((count, n), dtype=torch.bool, device=dev)
        if causal:
            see = t <= p
            if window:
                see = see & ((t > p - window) | (t < sink))
        for h in range(H):
            keys, there = values(c, "k", b, h // (H // Hkv), n)
            vals, _ = values(c, "v", b, h // (H // Hkv), n)
            s_see = see & there
            some = s_see.any(1)
            if not some.any():
                out[b, h, :count], lse[b, h, :count] = 0, -math.inf
                continue
            keys = torch.where(s_see.any(0)[:, None], keys, 0.0)                # (what no query sees may be anything)
            s = (q[b, h, :count] @ keys.t().contiguous() * scale).masked_fill(~s_see, -math.inf)
            z = torch.where(some, torch.logsumexp(s, 1), -math.inf)
            w = torch.where(s_see & some[:, None], torch.exp(s - z[:, None]), 0.0)
            seen_vals = torch.where(s_see.any(0)[:, None], vals, 0.0)
            bad = seen_vals.isnan()
            o = w @ torch.where(bad, 0.0, seen_vals)
            o = torch.where((s_see.double() @ bad.double()) > 0, math.nan, o)      # a NaN reaches those that see it
            out[b, h, :count], lse[b, h, :count] = o, z
            size = (q[b, h, :count].abs() @ keys.abs().t().contiguous() * scale).masked_fill(~s_see, 0.0).amax(1, keepdim=True)
            share = (d + 2) * F32 * size + 2.0 ** -20
            mean = w @ torch.where(bad, 0.0, seen_vals).abs()
            ob[b, h, :count] = HALF[dt] * o.abs().nan_to_num() + (HALF[dt] + 2 * share) * mean * 1.01 + TINY[dt] * (2 + s_see.sum(1, keepdim=True) * seen_vals.abs().nan_to_num().amax())
            lb[b, h, :count] = share[:, 0] + 2.0 ** -21 * (1 + torch.where(some, z.abs(), 0.0))
    return heads_first(out, layout), lse, heads_first(ob, layout), lb
