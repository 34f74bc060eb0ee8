"""Timing cases of the operators of a serving program whose cache is held in 8 bits and in pages: the norm of each head's queries and
keys with their rotation in the same pass (and its gradient, for training the weights), the append of new tokens to the cache, and attention over it.

A case is a plain dict (case["op"] is norm, grad, append or paged); prepare() makes what the caller has in hand, run() is one
call: the operator's plain form in elementary torch operations, or, where `own` is true, the framework's.

The cache: codes are e4m3, [pages, H_kv, page, d]; a block of 32 tokens of a page and head has one scale, a power of two (e8m0,
[pages, H_kv, page / 32]); a value is its code times the scale.  page_table [B, pages of a sequence] says where tokens are.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "fp16": torch.float16}
_F8, _E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
_CAP = {"bf16": 246, "fp16": 134}        # the largest scales, 2^119 and 2^7: no value of a code is beyond the type that it came from


def listed():
    return [
        # one new token for each of 16 sequences far into a long context: launch and host time are all there is
        _norm("norm_step", B=16, H=32, H_kv=8, N=1, far=32768),
        # a batch of prompts, queries and keys as a fused projection leaves them, grouped KV heads
        _norm("norm_prompts4k", B=4, H=32, H_kv=8, N=4096, layout="NHD", weights="f32"),
        # the gradient at a ragged length, 64-wide heads, half of each turned, neighbouring channels in pairs
        _norm("grad_ragged", op="grad", B=1, H=16, H_kv=16, N=3001, d=64, rot=32, dtype="fp16", interleaved=True),
        # a training step's gradient of two sequences of a fused projection
        _norm("grad_train4k", op="grad", B=2, H=32, H_kv=8, N=4096, layout="NHD", weights="f32"),
        # the new token of each of 32 sequences
        _append("append_step", B=32, H_kv=8, N=1, cap=8192),
        # up to five accepted tokens per sequence, 256-wide heads, small pages
        _append("append_tokens5_d256", B=6, H_kv=4, N=5, cap=1024, d=256, page=32, dtype="fp16", layout="NHD", ragged=True),
        # two prompts into an empty cache
        _append("append_prompt8k", B=2, H_kv=8, N=8192, cap=8192, layout="NHD"),
        # a handful of short conversations, 64-wide heads, one of them idle
        _paged("paged_small", B=4, H=8, H_kv=2, N=1, cap=512, d=64, dtype="fp16", page=32, idle=True),
        # a decode step over long caches
        _paged("paged_step32k", B=16, H=32, H_kv=8, N=1, cap=32768),
        # a decode step whose queries see the last 4096 tokens and the first 4
        _paged("paged_window4k", B=32, H=32, H_kv=8, N=1, cap=16384, window=4096, sink=4),
        # up to five proposed tokens per sequence, 256-wide heads, token-major queries, an odd window
        _paged("paged_tokens5_d256", B=6, H=16, H_kv=4, N=5, cap=5120, d=256, page=32, layout="NHD", ragged=True, window=3001, sink=33),
        # chunks of 512 tokens of two prompts over what is in the cache already
        _paged("paged_chunk512", B=2, H=32, H_kv=8, N=512, cap=16384, page=128),
    ]


def _named(name, c):
    if name:
        c["name"] = name
    return c


def _norm(name, **kw):
    c = dict(op="norm", B=1, H=32, H_kv=8, N=1, d=128, rot=0, dtype="bf16", layout="HND", weights="same", interleaved=False, far=1)
    c.update(kw)
    c["rot"] = c["rot"] or c["d"]
    return _named(name, c)


def _append(name, **kw):
    return _named(name, dict(dict(op="append", B=1, H_kv=8, N=1, cap=64, d=128, page=64, dtype="bf16", layout="HND", ragged=False), **kw))


def _paged(name, **kw):
    return _named(name, dict(dict(op="paged", B=1, H=32, H_kv=8, N=1, cap=64, d=128, page=64, dtype="bf16", layout="HND", ragged=False, idle=False,
                                  window=0, sink=0), **kw))


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["norm", "grad", "append", "paged", "paged", "paged"])
    d = rng.choice([64, 128, 128, 256])
    G, Hkv = rng.choice([1, 2, 4, 4, 8]), rng.choice([1, 2, 4, 8, 8, 12])
    c = dict(op=op, B=_log_int(rng, 1, 48), d=d, H_kv=Hkv, dtype=rng.choice(["bf16", "bf16", "fp16"]), layout=rng.choice(["HND", "NHD"]))
    if op in ("norm", "grad"):
        c.update(H=G * Hkv, N=_log_int(rng, 1, 20000), interleaved=rng.random() < 0.4, far=_log_int(rng, 1, 1000000), rot=rng.choice([d, d, d, d // 2, d // 4]),
                 weights=rng.choice(["same", "f32"]))
        while c["B"] * c["N"] * (c["H"] + Hkv) * d > (8 if op == "norm" else 4) * 10 ** 7:
            c["B"], c["N"] = max(1, c["B"] // 2), max(1, c["N"] * 2 // 3)
        return _norm("", **c)
    c["page"] = rng.choice([32, 64, 64, 128, 256])
    if op == "append":
        c["N"] = rng.choice([1, 1, 2, 5, _log_int(rng, 1, 10000), _log_int(rng, 1, 10000)])
        c["cap"] = c["N"] + _log_int(rng, 1, 8192)
        while c["B"] * c["cap"] * Hkv * d > 3 * 10 ** 7:
            c["B"], c["N"] = max(1, c["B"] // 2), max(1, c["N"] * 2 // 3)
            c["cap"] = max(c["N"], c["cap"] * 2 // 3)
        c["ragged"] = rng.random() < 0.5
        c["cap"] = -(-c["cap"] // c["page"]) * c["page"]
        return _append("", **c)
    c.update(H=G * Hkv, N=rng.choice([1, 1, 1, 1, 2, 3, 5, 8, _log_int(rng, 9, 600)]), cap=_log_int(rng, 32, 60000), ragged=rng.random() < 0.5, idle=rng.random() < 0.2)
    while c["B"] * Hkv * c["cap"] * d > 3 * 10 ** 8 or c["B"] * c["H"] * c["N"] * c["cap"] > 3 * 10 ** 8:
        c["B"], c["cap"] = max(1, c["B"] // 2), max(32, c["cap"] * 2 // 3)
        c["N"] = max(1, c["N"] * 4 // 5)
    c["cap"] = -(-max(c["cap"], c["N"]) // c["page"]) * c["page"]
    if rng.random() < 0.5:
        c.update(window=_log_int(rng, 1, 8192), sink=rng.choice([0, 0, 1, 4, 4, 64, 100]))
    return _paged("", **c)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _randn(g, shape, dt, std=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dt)


def _tokens(g, case, heads, std=1.0):
    """Rows of `heads` kinds of heads; token-major ones are views of one buffer, as a fused projection leaves them."""
    B, N, d, dt = case["B"], case["N"], case["d"], _T[case["dtype"]]
    if case["layout"] == "HND":
        return [_randn(g, (B, h, N, d), dt, std) for h in heads]
    return list(_randn(g, (B, N, sum(heads), d), dt, std).split(heads, dim=2))


def _like(x):
    """Room for a result laid out like x, a view of a larger buffer or not."""
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")


def _lens(g, case, least):
    """Lengths of caches of `cap` tokens: one full, the others from a quarter up, `least` [B] at least."""
    n = case["cap"]
    x = torch.rand(case["B"], generator=g, device="cuda").mul_(0.75).add_(0.25).mul_(n).to(torch.int32)
    x = torch.maximum(x, least)
    x[torch.randint(case["B"], (), generator=g, device="cuda")] = n
    return x


def _counts(g, case):
    """How many of the N tokens of a call each sequence has."""
    if not case["ragged"]:
        return None
    return torch.randint(1, case["N"] + 1, (case["B"],), generator=g, device="cuda").to(torch.int32)


def _pages(g, case):
    """A page table over a pool somewhat larger than what it names, and the pool's size."""
    of_one = case["cap"] // case["page"]
    used = case["B"] * of_one
    pool = used + used // 16 + 1
    return torch.randperm(pool, generator=g, device="cuda")[:used].to(torch.int32).reshape(case["B"], of_one), pool


def _quantized(g, case, pool):
    """A pool of random keys or values as an append leaves it, made page by page."""
    Hkv, page, d = case["H_kv"], case["page"], case["d"]
    codes = torch.empty((pool, Hkv, page, d), dtype=_F8, device="cuda")
    scale = torch.empty((pool, Hkv, page // 32), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (Hkv * page * d))
    for i in range(0, pool, step):
        n = min(step, pool - i)
        x = torch.randn((n, Hkv, page // 32, 32, d), generator=g, device="cuda")
        x *= torch.rand((n, Hkv, page // 32, 1, 1), generator=g, device="cuda").mul_(2.0).add_(0.5)       # blocks differ in size
        e = _scale_of(x.abs().amax((-1, -2)), case)
        codes[i:i + n] = (x / _two(e)[..., None, None]).to(_F8).reshape(n, Hkv, page, d)
        scale[i:i + n] = e.to(torch.uint8)
    return codes, scale.view(_E8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt, B, Hkv, d = _T[case["dtype"]], case["B"], case["H_kv"], case["d"]
    s = dict(case=case)
    if case["op"] in ("norm", "grad"):
        s["q"], s["k"] = _tokens(g, case, [case["H"], Hkv], 3.0)
        wt = torch.float32 if case["weights"] == "f32" else dt
        s["q_weight"], s["k_weight"] = (torch.randn(d, generator=g, device="cuda").mul_(0.2).add_(1.0).to(wt) for _ in range(2))
        s["inv_freq"] = 500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
        first = torch.randint(case["far"], (B, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(case["N"], device="cuda")).to(torch.int32)
        if case["op"] == "grad":
            s["dq_out"], s["dk_out"] = _tokens(g, case, [case["H"], Hkv])
        s["q_to"], s["k_to"] = _like(s["q"]), _like(s["k"])
        return s
    s["page_table"], pool = _pages(g, case)
    counts = _counts(g, case)
    s["counts"] = counts
    least = counts if counts is not None else torch.full((B,), case["N"], dtype=torch.int32, device="cuda")
    s["kv_lens"] = _lens(g, case, least)
    s["k_cache"], s["k_scale"] = _quantized(g, case, pool)
    s["v_cache"], s["v_scale"] = _quantized(g, case, pool)
    if case["op"] == "append":
        s["k"], s["v"] = _tokens(g, case, [Hkv, Hkv], 2.0)
        return s
    if case["idle"] and B > 1:
        s["kv_lens"][torch.randint(B, (), generator=g, device="cuda")] = 0
    s["q"] = _randn(g, (B, case["N"], case["H"], d) if case["layout"] == "NHD" else (B, case["H"], case["N"], d), dt, 2.0)
    s["out"] = torch.zeros_like(s["q"])
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _scale_of(most, case):
    """The exponent byte of the smallest power of two of which 448 times is `most` or more; 2^-64 at least."""
    bits = most.float().view(torch.int32)
    e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000).int()
    return e.clamp(63, _CAP[case["dtype"]])


def _two(e):
    """2^(e - 127), 1 <= e <= 254."""
    return (e.int() << 23).view(torch.float32)


def _turns(s):
    """Cosine and sine of every token and pair, to be used with rows of the case's layout."""
    case = s["case"]
    angle = s["positions"].double()[..., None] * s["inv_freq"]
    at = 2 if case["layout"] == "NHD" else 1
    return angle.cos().float().unsqueeze(at), angle.sin().float().unsqueeze(at)


def _rotate(case, x, cos, sin):
    r = case["rot"]
    y = x.clone()
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * cos - b * sin, b * cos + a * sin
    return y


def _norm_plain(s):
    case = s["case"]
    cos, sin = _turns(s)
    def of(x, w):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        return _rotate(case, y, cos, sin).to(s["q"].dtype)
    return of(s["q"], s["q_weight"]), of(s["k"], s["k_weight"])


def _grad_plain(s):
    case = s["case"]
    cos, sin = _turns(s)
    def of(x, w, dy):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        n = x * r
        dy = _rotate(case, dy.float(), cos, -sin)
        dw = (dy * n).sum((0, 1, 2))
        dn = dy * w.float()
        return (r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(s["q"].dtype), dw
    dq, dqw = of(s["q"], s["q_weight"], s["dq_out"])
    dk, dkw = of(s["k"], s["k_weight"], s["dk_out"])
    return dq, dk, dqw, dkw


def _append_one(s, new, cache, scale):
    case = s["case"]
    B, Hkv, N, d, page = (case[n] for n in ("B", "H_kv", "N", "d", "page"))
    new = (new.transpose(1, 2) if case["layout"] == "NHD" else new).float()
    counts = s["counts"].long() if s["counts"] is not None else torch.full((B,), N, device="cuda")
    first = s["kv_lens"].long() - counts                                    # where the new tokens start
    # The blocks that they touch, as [B, H_kv, blocks, 32, d], with what is there before them
    blocks = (N + 62) // 32
    token = (first // 32 * 32)[:, None] + torch.arange(blocks * 32, device="cuda")
    at = token - first[:, None]                                             # which new token it is
    is_new = (at >= 0) & (at < counts[:, None])
    pages = s["page_table"].long().gather(1, (token // page).clamp(max=s["page_table"].shape[1] - 1))
    old = cache.view(torch.uint8)[pages, :, token % page].view(_F8).float().transpose(1, 2)       # [B, H_kv, 32 blocks, d]
    block = pages[:, ::32], (token % page // 32)[:, ::32]
    e_old = scale.view(torch.uint8)[block[0], :, block[1]].int().transpose(1, 2)                  # [B, H_kv, blocks]
    x = new.gather(2, at.clamp(0, N - 1)[:, None, :, None].expand(-1, Hkv, -1, d))
    x = torch.where(is_new[:, None, :, None], x, 0.0).reshape(B, Hkv, blocks, 32, d)
    touched = is_new.reshape(B, 1, blocks, 32).any(-1)
    kept = ((at < 0) & (token >= 0)).reshape(B, 1, blocks, 32)[..., 0]      # blocks that hold earlier tokens
    e = _scale_of(x.abs().amax((-1, -2)), case)
    e = torch.where(kept, torch.maximum(e, e_old), e)
    codes = (x / _two(e)[..., None, None]).clamp(-448.0, 448.0).to(_F8)
    again = (old.reshape(x.shape) * _two(e_old - e + 127)[..., None, None]).to(_F8)
    put = is_new.reshape(B, 1, blocks, 32, 1)
    before = ((at < 0) & (token >= 0)).reshape(B, 1, blocks, 32, 1) & touched[..., None, None]
    codes = torch.where(put, codes.view(torch.uint8), torch.where(before, again.view(torch.uint8), old.to(_F8).reshape(x.shape).view(torch.uint8)))
    b, j = touched[:, 0].nonzero(as_tuple=True)
    page_of, in_page = block[0][b, j], block[1][b, j]
    cache.view(torch.uint8).unflatten(2, (-1, 32))[page_of, :, in_page] = codes[b, :, j]
    scale.view(torch.uint8)[page_of, :, in_page] = e[b, :, j].to(torch.uint8)


def _append_plain(s):
    _append_one(s, s["k"], s["k_cache"], s["k_scale"])
    _append_one(s, s["v"], s["v_cache"], s["v_scale"])
    return s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]


def _values(s, codes, scale):
    """All tokens of every sequence, [B, H_kv, cap, d] in 32 bits."""
    case = s["case"]
    at = s["page_table"].long()
    x = codes.view(torch.uint8)[at].view(_F8).float().unflatten(3, (-1, 32))
    x *= _two(scale.view(torch.uint8)[at])[..., None, None]
    return x.transpose(1, 2).reshape(case["B"], case["H_kv"], case["cap"], case["d"])


def _paged_plain(s):
    case = s["case"]
    B, H, Hkv, N, d = (case[n] for n in ("B", "H", "H_kv", "N", "d"))
    q = (s["q"].transpose(1, 2) if case["layout"] == "NHD" else s["q"]).float().reshape(B, Hkv, -1, d)
    x = torch.matmul(q, _values(s, s["k_cache"], s["k_scale"]).transpose(2, 3)).mul_(1 / math.sqrt(d))
    lens = s["kv_lens"].long()
    counts = s["counts"].long() if s["counts"] is not None else torch.full_like(lens, N)
    r, t = torch.arange(N, device="cuda"), torch.arange(case["cap"], device="cuda")
    last = (lens - counts).clamp(min=0)[:, None, None] + r[:, None]         # [B, N, 1]
    seen = (t <= last) & (t < lens[:, None, None])
    if case["window"]:
        seen &= (t > last - case["window"]) | (t < case["sink"])
    x = x.reshape(B, Hkv, -1, N, case["cap"]).masked_fill_(~seen[:, None, None], -math.inf).reshape(B, Hkv, -1, case["cap"])
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = (torch.matmul(x, _values(s, s["v_cache"], s["v_scale"])) / total.clamp(min=1e-30)).reshape(B, H, N, d).to(s["q"].dtype)
    lse = (m + total.log()).reshape(B, H, N)
    there = r < counts[:, None]                                             # queries behind a sequence's last are left as they were
    o = o.transpose(1, 2) if case["layout"] == "NHD" else o
    o = torch.where(there[:, :, None, None] if case["layout"] == "NHD" else there[:, None, :, None], o, s["out"])
    return o.contiguous(), torch.where(there[:, None], lse, 0.0)


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    return {"norm": _norm_plain, "grad": _grad_plain, "append": _append_plain, "paged": _paged_plain}[s["case"]["op"]](s)


def _own(s):
    import paper_2411_10958_amd as sage
    case = s["case"]
    op = case["op"]
    if op == "norm":
        return sage.sage_qk_norm_rope(s["q"], s["k"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, positions=s["positions"],
                                      interleaved=case["interleaved"], layout=case["layout"], q_out=s["q_to"], k_out=s["k_to"])
    if op == "grad":
        return sage.sage_qk_norm_rope_bwd(s["dq_out"], s["q"], s["dk_out"], s["k"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                                          positions=s["positions"], interleaved=case["interleaved"], layout=case["layout"], dq=s["q_to"], dk=s["k_to"])
    if op == "append":
        sage.sage_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["page_table"], s["kv_lens"], new_lens=s["counts"],
                               layout=case["layout"])
        return s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]
    return sage.sage_attn_paged(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["page_table"], kv_lens=s["kv_lens"], q_lens=s["counts"],
                                out=s["out"], window=case["window"], sink=case["sink"], layout=case["layout"], return_lse=True)


def work(case):
    """Inputs read once, outputs written once.  The lengths of caches are drawn with the inputs: on average five eighths of the
    capacity are used, one sequence's all of it; tokens that no query sees are not read.  Of N tokens of a ragged call (N + 1) / 2 are there."""
    B, Hkv, N, d = case["B"], case["H_kv"], case["N"], case["d"]
    if case["op"] in ("norm", "grad"):
        values = B * N * (case["H"] + Hkv) * d
        weights = 2.0 * d * (4 if case["weights"] == "f32" else 2)
        if case["op"] == "norm":
            return {"bytes": 4.0 * values + 4.0 * B * N + 4.0 * case["rot"] + weights, "flops": 4.0 * values + 3.0 * values * case["rot"] / d}
        return {"bytes": 6.0 * values + 4.0 * B * N + 4.0 * case["rot"] + weights + 8.0 * d, "flops": 11.0 * values + 3.0 * values * case["rot"] / d}
    n = (N + 1) / 2 if case["ragged"] else N
    if case["op"] == "append":
        tokens = B * n * Hkv * 2
        return {"bytes": tokens * (3.0 * d + 1 / 32), "flops": 2.0 * tokens * d}
    H = case["H"]
    used = [case["cap"]] + [0.625 * case["cap"]] * (B - 1)
    keys = pairs = 0.0
    for x in used:
        if case["window"]:
            keys += min(x, case["window"] + case["sink"] + n - 1)
            pairs += n * min(x, case["window"] + case["sink"])
        else:
            keys += x
            pairs += n * (x - (n - 1) / 2)
    if case["idle"] and B > 1:
        keys, pairs = keys * (B - 1) / B, pairs * (B - 1) / B
    return {"bytes": 2.0 * keys * Hkv * (d + 1 / 32) + 4.0 * B * H * n * d + 4.0 * B * H * n, "flops": 4.0 * d * H * pairs}


# ---- 64 bits, from the definitions --------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return tuple(_norm64(case, s, s[n], s[n + "_weight"])[0] for n in "qk")
    if case["op"] == "grad":
        q, k = (_norm64(case, s, s[n], s[n + "_weight"], s["d%s_out" % n]) for n in "qk")
        return q[0], k[0], q[1], k[1]
    if case["op"] == "append":
        return _append64(case, s, "k") + _append64(case, s, "v")
    return _paged64(case, s)


def _norm64(case, s, x, w, dy=None):
    """Pairs as complex numbers, turned by exp(i p f); the gradient by torch's own rules of differentiation."""
    r = case["rot"]
    x, w = x.double().requires_grad_(dy is not None), w.double().requires_grad_(dy is not None)
    p = s["positions"].double()
    p = p[:, :, None, None] if case["layout"] == "NHD" else p[:, None, :, None]
    angle = p * s["inv_freq"]
    turn = torch.polar(torch.ones_like(angle), angle)
    n = x / (x.square().sum(-1, keepdim=True) / case["d"] + 1e-6).sqrt() * w
    pairs = (n[..., :r].unflatten(-1, (r // 2, 2)) if case["interleaved"] else n[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)).contiguous()
    y = torch.view_as_real(torch.view_as_complex(pairs) * turn)
    y = torch.cat([(y if case["interleaved"] else y.transpose(-1, -2)).flatten(-2), n[..., r:]], -1)
    return (y,) if dy is None else torch.autograd.grad(y, (x, w), dy.double())


def _two64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round64(y):
    """To the nearest of e4m3's numbers, ties to the even one."""
    _, e = torch.frexp(y)
    step = _two64((e - 4).clamp(min=-9))
    return ((y / step).round() * step).clamp(-448, 448)


def _append64(case, s, name):
    """Sequence by sequence, block by block."""
    cache, scale = s[name + "_cache"].double(), s[name + "_scale"].double()
    new, page = s[name].double(), case["page"]
    most = 7 if case["dtype"] == "fp16" else 119
    for b in range(case["B"]):
        n = case["N"] if s["counts"] is None else int(s["counts"][b])
        first = int(s["kv_lens"][b]) - n
        for start in range(first // 32 * 32, first + n, 32):
            at, j = int(s["page_table"][b, start // page]), start % page // 32
            lo, hi = max(start, first), min(start + 32, first + n)
            x = new[b, lo - first:hi - first].transpose(0, 1) if case["layout"] == "NHD" else new[b, :, lo - first:hi - first]      # [H_kv, tokens, d]
            f, e = torch.frexp(x.abs().amax((1, 2)))
            e = (e - 9 + (f > 0.875).int()).clamp(-64, most)
            two = _two64(e)
            block = cache[at, :, 32 * j:32 * j + 32]
            if lo > start:
                two = torch.maximum(two, scale[at, :, j])
                block[:, :lo - start] = _round64(block[:, :lo - start] * (scale[at, :, j] / two)[:, None, None])
            block[:, lo - start:hi - start] = _round64(x / two[:, None, None])
            scale[at, :, j] = two
    return cache, scale


def _paged64(case, s):
    B, H, Hkv, N, d, page = (case[n] for n in ("B", "H", "H_kv", "N", "d", "page"))
    if B * H * N * case["cap"] * d > 1e12:
        return None
    nhd = case["layout"] == "NHD"
    out, lse = s["out"].double(), torch.zeros((B, H, N), dtype=torch.float64, device="cuda")
    for b in range(B):
        n, count = int(s["kv_lens"][b]), N if s["counts"] is None else int(s["counts"][b])
        t = torch.arange(n, device="cuda")
        at = s["page_table"][b].long()[t // page]
        p = max(n - count, 0) + torch.arange(count, device="cuda")[:, None]
        hidden = t > p
        if case["window"]:
            hidden |= (p - t >= case["window"]) & (t >= case["sink"])
        for h in range(Hkv):
            keys, values = (s[x + "_cache"].view(torch.uint8)[at, h, t % page].view(_F8).double() * s[x + "_scale"].view(torch.uint8)[at, h, t % page // 32].view(_E8).double()[:, None]
                            for x in "kv")
            for i in range(h * (H // Hkv), (h + 1) * (H // Hkv)):
                q = (s["q"][b, :count, i] if nhd else s["q"][b, i, :count]).double()
                x = (q @ keys.t().contiguous() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                z = torch.logsumexp(x, -1) if n else torch.full((count,), -math.inf, dtype=torch.float64, device="cuda")
                o = torch.exp(x - z[:, None]).nan_to_num(0.0) @ values
                (out[b, :count, i] if nhd else out[b, i, :count])[:] = o
                lse[b, i, :count] = z
    return out, lse
