"""The operators around attention in float64, from their definitions, and how far a kernel may be from them.

A rounding to a 16-bit type is off by at most half a step, HALF[dtype] of the value; FP32 is 2^-24.  The bounds returned beside the
results add up such roundings in the worst case, so no measured figure is in them."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}          # half a step of the smallest numbers
F32 = 2.0 ** -24


def heads_first(x, layout):
    return x.transpose(-2, -3) if layout == "NHD" else x


def to_layout(x, layout):
    return x.transpose(1, 2).contiguous() if layout == "NHD" else x.contiguous()


def rope(x, inv_freq, positions, interleaved, inverse, scale, layout):
    """x [B, heads, N, d] in `layout`; positions [N] or [B, N] (whole numbers).  Returns the result and its bound: half a step of
    the output, and for each of the two products and their sum the rounding of the cosine (two units), the scale, the product
    and the sum: less than 8 units of 2^-24 of |a| + |b|."""
    h = heads_first(x, layout).double()
    r = 2 * inv_freq.numel()
    p = positions.double()
    p = p[None, :] if p.dim() == 1 else p
    angle = (p[:, None, :, None] * inv_freq.double()) * (-1 if inverse else 1)
    c, s = angle.cos() * scale, angle.sin() * scale
    y, bound = h.clone(), torch.zeros_like(h)
    ia = torch.arange(0, r, 2) if interleaved else torch.arange(r // 2)
    ib = ia + (1 if interleaved else r // 2)
    a, b = h[..., ia], h[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    room = HALF[x.dtype] * y.abs() + TINY[x.dtype]
    fp32 = 8 * F32 * abs(scale) * (a.abs() + b.abs())
    bound[..., ia], bound[..., ib] = room[..., ia] + fp32, room[..., ib] + fp32
    return heads_first(y, layout), heads_first(bound, layout)


def _visible(n, nk, length, causal, device):
    """[n, nk]: whether query r sees key t of a cache with `length` tokens in use."""
    t = torch.arange(nk, device=device)
    see = (t < length).expand(n, nk)
    return see & (t <= torch.arange(n, device=device)[:, None] + max(length - n, 0)) if causal else see


def shared_prefix(q, kp, vp, k, v, lens, causal, sm_scale, layout):
    """out, lse in float64 and their bounds.  The weights P are rounded to the type of V (half a step, or half of the smallest number)
    and so is the output; a score is off by d + 2 FP32 roundings of sum |q| |k|, which moves a weight by that share."""
    dt, dev = q.dtype, q.device
    q = heads_first(q, layout).double()
    B, H, N, d = q.shape
    kp, vp, k, v = (None if x is None else heads_first(x, layout).double() for x in (kp, vp, k, v))
    Hkv = (kp.shape[0] if kp is not None else k.shape[1])
    scale = sm_scale if sm_scale > 0 else 1 / math.sqrt(d)
    out, lse = torch.zeros_like(q), torch.full((B, H, N), -math.inf, dtype=torch.float64, device=dev)
    ob, lb = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n = (k.shape[2] if k is not None else 0) if lens is None else min(max(int(lens[b]), 0), k.shape[2])
        for h in range(H):
            g = h // (H // Hkv)
            keys = torch.cat([x for x in (kp[g] if kp is not None else None, k[b, g, :n] if k is not None else None) if x is not None])
            vals = torch.cat([x for x in (vp[g] if vp is not None else None, v[b, g, :n] if k is not None else None) if x is not None])
            P = kp.shape[1] if kp is not None else 0
            if len(keys) == 0:
                continue
            see = torch.cat([torch.ones(N, P, dtype=torch.bool, device=dev), _visible(N, n, n, causal, dev)], 1)
            s = (q[b, h] @ keys.t().contiguous() * scale).masked_fill(~see, -math.inf)
            some = see.any(1)
            lse[b, h] = torch.logsumexp(s, 1)
            p = torch.where(see & some[:, None], torch.exp(s - lse[b, h][:, None]), 0.0)
            vals = torch.where(see.any(0)[:, None], vals, 0.0)
            out[b, h] = p @ vals
            size = (q[b, h].abs() @ keys.abs().t().contiguous() * scale).masked_fill(~see, 0.0).amax(1, keepdim=True)
            share = (d + 2) * F32 * size + 2.0 ** -20
            mean = p @ vals.abs()
            ob[b, h] = HALF[dt] * out[b, h].abs() + (HALF[dt] + 2 * share) * mean * 1.01 + TINY[dt] * (1 + see.sum(1, keepdim=True) * vals.abs().amax())
            lb[b, h] = share[:, 0] + 2.0 ** -21 * (1 + torch.where(some, lse[b, h].abs(), 0.0))
    return heads_first(out, layout), lse, heads_first(ob, layout), lb


def key_weights(q, k, lse, w_in, w_old, lens, causal, sm_scale, layout):
    """Weights in float64 and their bound: the score as above, the exponent's other terms (lse log2 e, the sum) three roundings of
    their size, the exponential two, the sum of R weights and w_in R + 1."""
    q, k = heads_first(q, layout).double(), heads_first(k, layout).double()
    B, H, N, d = q.shape
    Hkv, nk = k.shape[1], k.shape[2]
    scale = sm_scale if sm_scale > 0 else 1 / math.sqrt(d)
    w, bound = w_old.double().clone(), torch.zeros(w_old.shape, dtype=torch.float64, device=q.device)
    for b in range(B):
        n = nk if lens is None else min(max(int(lens[b]), 0), nk)
        see = _visible(N, nk, n, causal, q.device)[:, :n]
        for g in range(Hkv):
            total = torch.zeros(n, dtype=torch.float64, device=q.device) if w_in is None else w_in[b, g, :n].double().clone()
            off = total.abs() * F32
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                L = lse[b, h].double()[:, None]
                s = q[b, h] @ k[b, g, :n].t().contiguous() * scale
                p = torch.where(see & (L > -math.inf), torch.exp(s - L), 0.0)
                size = q[b, h].abs() @ k[b, g, :n].abs().t().contiguous() * scale
                total += p.sum(0)
                off += (torch.where(p > 0, p * ((d + 2) * F32 * size + 6 * F32 * (s.abs() + L.abs()) + 4 * F32), 0.0)).sum(0)
            w[b, g, :n] = total
            bound[b, g, :n] = off + (N * (H // Hkv) + 1) * F32 * total.abs() + 1e-37
    return w, bound


def evict(k, v, w, keep, sink, recent, lens, layout):
    """Per sequence and KV head, the indices kept (lists)."""
    B, Hkv, nk = w.shape
    res = []
    for b in range(B):
        n = nk if lens is None else min(max(int(lens[b]), 0), nk)
        row = []
        for g in range(Hkv):
            x = w[b, g, :n].double().cpu().tolist()
            if n <= keep:
                row.append(list(range(n)))
                continue
            mid = sorted(range(sink, n - recent), key=lambda t: ((0, 0.0) if x[t] != x[t] else (-1, -x[t]), t))
            row.append(sorted(list(range(sink)) + mid[:keep - sink - recent] + list(range(n - recent, n))))
        res.append(row)
    return res


def check(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    got = got.double()
    same = (got == want) | (got.isnan() & want.isnan())
    over = torch.where(same, 0.0, (got - want).abs() / bound.clamp(min=1e-300))
    worst = over.nan_to_num(nan=math.inf).max().item() if over.numel() else 0.0
    assert worst <= 1, f"{name}: {worst:.3g} of the bound"
