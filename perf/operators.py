"""Timing cases of the operators around the attention calls of a serving program: rotary positions of queries and keys,
16-bit attention of a batch that shares a prefix, the attention weight that keys have received, and the eviction of the
others from a cache.

A case is a plain dict (case["op"] is rope, shared, weights or evict); prepare() makes what the caller has in hand,
run() is one call: the operator's plain form in elementary torch operations, or, where `own` is true, the framework's.
"""
import math

import torch

own = False

_T = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one new token for each of 16 sequences far into a long context: launch and host time are all there is
        _rope("rope_step", B=16, H=32, H_kv=8, N=1, far=32768),
        # a batch of prompts, token-major as a fused projection leaves it, grouped KV heads
        _rope("rope_prompts4k", B=4, H=32, H_kv=8, N=4096, layout="NHD", far=1),
        # the gradient of a partial interleaved rotation at the ragged length of a video model
        _rope("rope_grad17k", B=2, H=48, H_kv=48, N=17776, d=64, rot=32, dtype="fp16", interleaved=True, inverse=True, far=1),
        # a handful of short questions to one short system prompt
        _shared("shared_small", B=4, H=8, H_kv=2, N=1, P=300, N_kv=50, d=64, dtype="fp16"),
        # a serving step: 32 conversations over one 8k prompt, each with up to 1k tokens of its own
        _shared("shared_step8k", B=32, H=32, H_kv=8, N=1, P=8192, N_kv=1024),
        # five proposed tokens per sequence, 256-wide heads, token-major caches
        _shared("shared_tokens5_d256", B=6, H=16, H_kv=4, N=5, P=5003, N_kv=777, d=256, layout="NHD"),
        # a large batch over a long document
        _shared("shared_step32k", B=64, H=32, H_kv=8, N=1, P=32768, N_kv=4096),
        # the weight that the keys of a prompt have received from all of its queries
        _weights("weights_prompt8k", B=1, H=32, H_kv=8, N=8192, N_kv=8192, d=128, ragged=False),
        # a chunk of 512 new queries against a 16k cache, 64-wide heads, added to what the keys have
        _weights("weights_chunk512", B=2, H=16, H_kv=16, N=512, N_kv=16384, d=64, dtype="fp16", layout="NHD", added=True),
        # one decode step against a 32k cache of four sequences, added to what the keys have
        _weights("weights_step32k", B=4, H=32, H_kv=8, N=1, N_kv=32768, d=128, added=True),
        # a small cache cut to a third, one of whose sequences is shorter than what is kept
        _evict("evict_small", B=2, H_kv=2, N_kv=700, keep=256, d=64, dtype="fp16", layout="NHD", sink=4, recent=32),
        # long caches of four sequences cut to half
        _evict("evict_32k", B=4, H_kv=8, N_kv=32768, keep=16384, d=128, sink=4, recent=1024),
    ]


def _named(name, c):
    if name:
        c["name"] = name
    return c


def _rope(name, **kw):
    c = dict(op="rope", B=1, H=32, H_kv=8, N=1, d=128, rot=0, dtype="bf16", layout="HND", interleaved=False, inverse=False, far=1, factor=8.0)
    c.update(kw)
    c["rot"] = c["rot"] or c["d"]
    return _named(name, c)


def _shared(name, **kw):
    return _named(name, dict(dict(op="shared", B=1, H=32, H_kv=8, N=1, P=0, N_kv=1, d=128, dtype="bf16", layout="HND"), **kw))


def _weights(name, **kw):
    return _named(name, dict(dict(op="weights", B=1, H=32, H_kv=8, N=1, N_kv=1, d=128, dtype="bf16", layout="HND", causal=True, ragged=True, added=False), **kw))


def _evict(name, **kw):
    return _named(name, dict(dict(op="evict", B=1, H_kv=8, N_kv=1, keep=1, d=128, dtype="bf16", layout="HND", sink=0, recent=0), **kw))


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["rope", "shared", "shared", "weights", "weights", "evict"])
    d = rng.choice([64, 128, 128, 256])
    G, Hkv = rng.choice([1, 2, 4, 4, 8]), rng.choice([1, 2, 4, 8, 8, 12])
    c = dict(d=d, H_kv=Hkv, dtype=rng.choice(["bf16", "bf16", "fp16"]), layout=rng.choice(["HND", "NHD"]))
    if op == "rope":
        c.update(H=G * Hkv, B=_log_int(rng, 1, 32), N=_log_int(rng, 1, 20000), interleaved=rng.random() < 0.5,
                 inverse=rng.random() < 0.3, far=_log_int(rng, 1, 1000000), rot=rng.choice([d, d, d // 2, d // 4, d - 8]))
        while c["B"] * c["N"] * (c["H"] + Hkv) * d > 2 * 10 ** 8:
            c["B"], c["N"] = max(1, c["B"] // 2), max(1, c["N"] * 2 // 3)
        return _rope("", **c)
    if op == "shared":
        c.update(H=G * Hkv, B=_log_int(rng, 1, 96), N=rng.choice([1, 1, 1, 2, 3, 5, 8]), P=_log_int(rng, 1, 40000))
        c["N_kv"] = _log_int(rng, c["N"], 6000)                              # the new tokens' own keys are in the cache
        while c["B"] * Hkv * c["N_kv"] * d > 2.5 * 10 ** 8 or c["B"] * c["H"] * c["N"] * (c["P"] + c["N_kv"]) * d > 8 * 10 ** 9:
            c["B"], c["P"], c["N_kv"] = max(1, c["B"] // 2), max(1, c["P"] * 2 // 3), max(c["N"], c["N_kv"] * 2 // 3)
        return _shared("", **c)
    if op == "weights":
        N = rng.choice([1, 1, 2, 5, _log_int(rng, 16, 600), _log_int(rng, 16, 600), _log_int(rng, 600, 6000)])
        c.update(H=G * Hkv, B=_log_int(rng, 1, 16), N=N, N_kv=N + _log_int(rng, 1, 30000) if rng.random() < 0.7 else N, causal=rng.random() < 0.8,
                 ragged=rng.random() < 0.5, added=rng.random() < 0.5)
        while c["B"] * c["H"] * N * c["N_kv"] > 10 ** 9 or c["B"] * Hkv * c["N_kv"] * d > 3 * 10 ** 8:
            c["B"], c["N_kv"] = max(1, c["B"] // 2), max(N, c["N_kv"] * 2 // 3)
            if c["B"] == 1 and c["N_kv"] == N:
                c["N"] = N = max(1, N * 2 // 3)
                c["N_kv"] = N
        return _weights("", **c)
    n = _log_int(rng, 2, 100000)
    keep = max(1, int(n * rng.uniform(0.1, 0.9)))
    sink = rng.randint(0, min(8, keep))
    c.update(B=_log_int(rng, 1, 16), N_kv=n, keep=keep, sink=sink, recent=rng.randint(0, (keep - sink) // 2))
    while c["B"] * Hkv * n * d > 2 * 10 ** 8 and c["B"] > 1:
        c["B"] //= 2
    return _evict("", **c)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _shape(case, heads, tokens):
    B, d = case["B"], case["d"]
    return (B, tokens, heads, d) if case["layout"] == "NHD" else (B, heads, tokens, d)


def _randn(g, shape, dt, std=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dt)


def _frequencies(rot, factor):
    """Base 500000, stretched by parts for a context `factor` times 8192: channels that turn less than once in it are slowed
    down by the factor, those that turn over four times are left."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    keep = ((8192 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
    return f * (keep + (1 - keep) / factor)


def _lens(g, case, least=1):
    """Lengths used of caches of N_kv tokens: one full, the others from a quarter up (never less than `least`)."""
    n = case["N_kv"]
    x = torch.rand(case["B"], generator=g, device="cuda").mul_(0.75).add_(0.25).mul_(n).to(torch.int32).clamp_(min=min(least, n), max=n)
    x[torch.randint(case["B"], (), generator=g, device="cuda")] = n
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = _T[case["dtype"]]
    Hkv = case["H_kv"]
    s = dict(case=case)
    if case["op"] == "rope":
        s.update(q=_randn(g, _shape(case, case["H"], case["N"]), dt, 2.0), k=_randn(g, _shape(case, Hkv, case["N"]), dt, 2.0),
                 inv_freq=_frequencies(case["rot"], case["factor"]), scale=0.1 * math.log(case["factor"]) + 1)
        first = torch.randint(case["far"], (case["B"], 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(case["N"], device="cuda")).to(torch.int32)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        return s
    N_kv = case["N_kv"]
    s["k"] = _randn(g, _shape(case, Hkv, N_kv), dt)
    if case["op"] == "evict":
        s["v"] = _randn(g, _shape(case, Hkv, N_kv), dt)
        s["kv_lens"] = _lens(g, case)
        w = torch.randn((case["B"], Hkv, N_kv), generator=g, device="cuda").mul_(2.0).exp_()
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.05, 0.0, w)     # keys that nothing attended to
        s["k_out"], s["v_out"] = (torch.zeros(_shape(case, Hkv, case["keep"]), dtype=dt, device="cuda") for _ in range(2))
        s["weights_out"] = torch.zeros((case["B"], Hkv, case["keep"]), device="cuda")
        s["kept"] = torch.zeros((case["B"], Hkv, case["keep"]), dtype=torch.int32, device="cuda")
        s["lens_out"] = torch.zeros(case["B"], dtype=torch.int32, device="cuda")
        return s
    s["q"] = _randn(g, _shape(case, case["H"], case["N"]), dt, 2.0)
    if case["op"] == "shared":
        s["v"] = _randn(g, _shape(case, Hkv, N_kv), dt)
        one = dict(case, B=1)
        s["k_prefix"], s["v_prefix"] = (_randn(g, _shape(one, Hkv, case["P"])[1:], dt) for _ in range(2))
        s["kv_lens"] = _lens(g, case, case["N"])
        s["out"] = torch.empty_like(s["q"])
        return s
    s["kv_lens"] = _lens(g, case, case["N"]) if case["ragged"] else None
    q, k = _grouped(case, s["q"]), _heads_first(case, s["k"])
    lse = [torch.logsumexp(_scores(case, q[b:b + 1, h:h + 1], k[b:b + 1, h:h + 1], s["kv_lens"][b:b + 1] if case["ragged"] else None), -1)
           for b in range(case["B"]) for h in range(Hkv)]
    s["lse"] = torch.cat(lse).reshape(case["B"], case["H"], case["N"]).contiguous()
    s["weights_in"] = torch.rand((case["B"], Hkv, N_kv), generator=g, device="cuda").mul_(4.0) if case["added"] else None
    s["weights"] = torch.zeros((case["B"], Hkv, N_kv), device="cuda")
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _heads_first(case, x):
    return x.float().transpose(1, 2) if case["layout"] == "NHD" else x.float()


def _grouped(case, q):
    """[B, H_kv, G N, d]: the queries of the heads that share a KV head."""
    q = _heads_first(case, q)
    return q.reshape(case["B"], case["H_kv"], -1, case["d"])


def _scores(case, q, k, kv_lens):
    """Scaled scores of grouped queries over a cache, -inf where a query does not see the key."""
    n, nk = case["N"], k.shape[2]
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1 / math.sqrt(case["d"]))
    t = torch.arange(nk, device="cuda")
    lens = torch.full((q.shape[0],), nk, device="cuda") if kv_lens is None else kv_lens.long()
    last = lens[:, None] - 1 + (torch.arange(n, device="cuda") - (n - 1) if case.get("causal", True) else torch.zeros(n, device="cuda", dtype=torch.long))
    last = last.repeat(1, q.shape[2] // n)[:, None, :, None]              # the last key that a query sees
    return s.masked_fill_(t > last, -math.inf)


def _rope_plain(s):
    case = s["case"]
    angle = s["positions"].double()[..., None] * s["inv_freq"]                      # [B, N, rot / 2]
    cos, sin = (angle.cos() * s["scale"]).float(), (angle.sin() * s["scale"]).float()
    if case["inverse"]:
        sin = -sin
    at = 2 if case["layout"] == "NHD" else 1
    cos, sin = cos.unsqueeze(at), sin.unsqueeze(at)
    return tuple(_rotate(case, s[n].float(), cos, sin).to(s[n].dtype) for n in "qk")


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


def _shared_plain(s):
    case = s["case"]
    B, H, Hkv, N, P, d = (case[n] for n in ("B", "H", "H_kv", "N", "P", "d"))
    q = _grouped(case, s["q"])
    own_scores = _scores(case, q, _heads_first(case, s["k"]), s["kv_lens"])
    kp, vp = (s[n].float().transpose(0, 1) if case["layout"] == "NHD" else s[n].float() for n in ("k_prefix", "v_prefix"))
    rows = q.transpose(0, 1).reshape(Hkv, -1, d)
    pre = torch.matmul(rows, kp.transpose(1, 2)).mul_(1 / math.sqrt(d)).reshape(Hkv, B, -1, P).transpose(0, 1)
    m = torch.maximum(own_scores.amax(-1, keepdim=True), pre.amax(-1, keepdim=True))
    e_own, e_pre = (own_scores - m).exp_(), (pre - m).exp_()
    total = e_own.sum(-1, keepdim=True) + e_pre.sum(-1, keepdim=True)
    o = torch.matmul(e_own, _heads_first(case, s["v"]))
    o += torch.matmul(e_pre.transpose(0, 1).reshape(Hkv, -1, P), vp).reshape(Hkv, B, -1, d).transpose(0, 1)
    o = (o / total).reshape(B, H, N, d).to(s["q"].dtype)
    lse = (m + total.log()).reshape(B, H, N)
    return (o.transpose(1, 2).contiguous() if case["layout"] == "NHD" else o), lse


def _weights_plain(s):
    case = s["case"]
    w = _scores(case, _grouped(case, s["q"]), _heads_first(case, s["k"]), s["kv_lens"])
    w = w.sub_(s["lse"].reshape(case["B"], case["H_kv"], -1, 1)).exp_().sum(2)
    if case["added"]:
        w = w + s["weights_in"]
    if s["kv_lens"] is None:
        return w
    return torch.where(torch.arange(case["N_kv"], device="cuda") < s["kv_lens"][:, None, None], w, s["weights"])


def _evict_plain(s):
    case = s["case"]
    n, keep = case["N_kv"], case["keep"]
    t, lens = torch.arange(n, device="cuda"), s["kv_lens"].long()[:, None, None]
    order = s["weights"].sort(dim=-1, descending=True, stable=True).indices
    rank = torch.where(t < lens, 1, 0) + torch.where((t < lens) & ((t < case["sink"]) | (t >= lens - case["recent"])), 1, 0)
    rank = rank.expand(case["B"], case["H_kv"], n).gather(-1, order)
    order = order.gather(-1, rank.sort(dim=-1, descending=True, stable=True).indices)[..., :keep]
    kept = torch.where(order < lens, order, n).sort(-1).values
    there, at = kept < n, kept.clamp(max=n - 1)
    rows = (lambda x: x.transpose(1, 2)) if case["layout"] == "NHD" else (lambda x: x)
    def moved(x, old):
        y = rows(x).gather(2, at[..., None].expand(-1, -1, -1, case["d"]))
        return rows(torch.where(there[..., None], y, rows(old))).contiguous()
    return (moved(s["k"], s["k_out"]), moved(s["v"], s["v_out"]), torch.where(there, s["weights"].gather(-1, at), s["weights_out"]),
            torch.where(there, at, s["kept"].long()).to(torch.int32), s["kv_lens"].clamp(max=keep))


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        return _own(s, case, op)
    return {"rope": _rope_plain, "shared": _shared_plain, "weights": _weights_plain, "evict": _evict_plain}[op](s)


def _own(s, case, op):
    import paper_2411_10958_amd as sage
    if op == "rope":
        return sage.sage_rope(s["q"], s["k"], s["inv_freq"], positions=s["positions"], interleaved=case["interleaved"], inverse=case["inverse"],
                              scale=s["scale"], layout=case["layout"], q_out=s["q_out"], k_out=s["k_out"])
    if op == "shared":
        return sage.sage_attn_shared_prefix(s["q"], s["k_prefix"], s["v_prefix"], s["k"], s["v"], kv_lens=s["kv_lens"], out=s["out"], causal=True,
                                            layout=case["layout"], return_lse=True)
    if op == "weights":
        return sage.sage_attn_key_weights(s["q"], s["k"], s["lse"], weights_in=s["weights_in"], weights=s["weights"], kv_lens=s["kv_lens"],
                                          causal=case["causal"], layout=case["layout"])
    return sage.sage_cache_evict(s["k"], s["v"], s["weights"], case["keep"], sink=case["sink"], recent=case["recent"], kv_lens=s["kv_lens"],
                                 layout=case["layout"], k_out=s["k_out"], v_out=s["v_out"], weights_out=s["weights_out"], kept=s["kept"],
                                 lens_out=s["lens_out"])


def work(case):
    """Inputs read once, outputs written once.  The lengths of ragged caches are drawn with the inputs: on average two thirds of the
    capacity are used, one sequence's all of it; keys past a length are neither read nor written."""
    B, Hkv, d = case["B"], case["H_kv"], case["d"]
    if case["op"] == "rope":
        values = B * case["N"] * (case["H"] + Hkv)
        return {"bytes": 4.0 * values * d + 4.0 * B * case["N"] + 4.0 * case["rot"], "flops": 3.0 * values * case["rot"]}
    used = (1 + (B - 1) * 0.625) * case["N_kv"]                              # tokens of all sequences
    if case["op"] == "evict":
        kept = min(used, B * case["keep"]) * Hkv
        return {"bytes": 4.0 * used * Hkv + kept * (8.0 * d + 8), "flops": used * Hkv}
    H, N = case["H"], case["N"]
    if case["op"] == "shared":
        return {"bytes": 4.0 * d * Hkv * (case["P"] + used) + 4.0 * B * H * N * d + 4.0 * B * H * N,
                "flops": 4.0 * d * H * N * (B * case["P"] + used - B * (N - 1) / 2)}
    if not case["ragged"]:
        used = B * case["N_kv"]
    pairs = H * N * (used - (B * (N - 1) / 2 if case["causal"] else 0))
    return {"bytes": 2.0 * d * (Hkv * used + B * H * N) + 4.0 * B * H * N + 4.0 * Hkv * used * (2 if case["added"] else 1), "flops": 2.0 * d * pairs}


# ---- 64 bits, from the definitions --------------------------------------------------------------------------------

def _visible64(case, b, kv_lens, r):
    """How many leading keys of its own cache query r of sequence b sees."""
    used = case["N_kv"] if kv_lens is None else kv_lens[b]
    return used - (case["N"] - 1 - r) if case.get("causal", True) else used


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return tuple(_rope64(case, s, s[n]) for n in "qk")
    B, Hkv = case["B"], case["H_kv"]
    lens = s["kv_lens"].tolist() if s["kv_lens"] is not None else None
    head = (lambda x, b, h: x[b, :, h]) if case["layout"] == "NHD" else (lambda x, b, h: x[b, h])
    if case["op"] == "evict":
        return _evict64(case, s, lens, head)
    G, N, nk = case["H"] // Hkv, case["N"], case["N_kv"]
    key = torch.arange(nk, device="cuda")
    if case["op"] == "weights":
        w = s["weights"].double()
        if B * case["H"] * N * nk * case["d"] > 2e12:
            return None
        for b in range(B):
            n = nk if lens is None else lens[b]
            see = torch.tensor([_visible64(case, b, lens, r) for r in range(N)], device="cuda")[:, None]
            for h in range(Hkv):
                w[b, h, :n] = s["weights_in"][b, h, :n].double() if case["added"] else 0
                for g in range(h * G, (h + 1) * G):
                    x = head(s["q"], b, g).double() @ head(s["k"], b, h).double().t().contiguous() / math.sqrt(case["d"])
                    x = torch.exp(x - s["lse"][b, g].double()[:, None])
                    w[b, h] += torch.where(key < see, x, 0.0).sum(0)
        return w
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty((B, case["H"], N), dtype=torch.float64, device="cuda")
    pre = (lambda x, h: x[:, h]) if case["layout"] == "NHD" else (lambda x, h: x[h])
    for h in range(Hkv):
        kp, vp = pre(s["k_prefix"], h).double(), pre(s["v_prefix"], h).double()
        for b in range(B):
            n = lens[b]
            keys = torch.cat([kp, head(s["k"], b, h)[:n].double()])
            values = torch.cat([vp, head(s["v"], b, h)[:n].double()])
            see = torch.tensor([case["P"] + _visible64(case, b, lens, r) for r in range(N)], device="cuda")[:, None]
            hidden = torch.arange(len(keys), device="cuda") >= see
            for g in range(h * G, (h + 1) * G):
                x = (head(s["q"], b, g).double() @ keys.t().contiguous() / math.sqrt(case["d"])).masked_fill(hidden, -math.inf)
                lse[b, g] = torch.logsumexp(x, -1)
                head(out, b, g)[:] = torch.exp(x - lse[b, g][:, None]) @ values
    return out, lse


def _rope64(case, s, x):
    """Pairs as complex numbers, turned by exp(i p f)."""
    r = case["rot"]
    x = x.double()
    p = s["positions"].double()
    p = p[:, :, None, None] if case["layout"] == "NHD" else p[:, None, :, None]
    turn = torch.polar(torch.full((), s["scale"], dtype=torch.float64, device="cuda"), p * s["inv_freq"] * (-1 if case["inverse"] else 1))
    pairs = (x[..., :r].unflatten(-1, (r // 2, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)).contiguous()
    y = torch.view_as_real(torch.view_as_complex(pairs) * turn)
    return torch.cat([(y if case["interleaved"] else y.transpose(-1, -2)).flatten(-2), x[..., r:]], -1)


def _evict64(case, s, lens, head):
    keep = case["keep"]
    k, v, w, kept, left = (s[n].clone() for n in ("k_out", "v_out", "weights_out", "kept", "lens_out"))
    for b, n in enumerate(lens):
        left[b] = min(n, keep)
        for h in range(case["H_kv"]):
            x = s["weights"][b, h, :n].double()
            x[:case["sink"]] = math.inf
            x[max(0, n - case["recent"]):] = math.inf
            at = (-x).sort(stable=True).indices[:keep].sort().values
            head(k, b, h)[:len(at)], head(v, b, h)[:len(at)] = head(s["k"], b, h)[at], head(s["v"], b, h)[at]
            w[b, h, :len(at)], kept[b, h, :len(at)] = s["weights"][b, h][at], at.to(torch.int32)
    return k.double(), v.double(), w.double(), kept, left
