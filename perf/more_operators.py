"""Timed cases of the serving step over an 8-bit cache, and of tokens' log probabilities with their gradient.

A step over the 8-bit cache is the step of the bf16 one with two other calls: append8 (norm + rotation of the new tokens,
keys and values quantised into their pages) and attention8 (the new tokens over the cache).  A page holds 64 tokens of a
KV head as e4m3 numbers under one scale, a power of two.  The logits that follow give the log probabilities of the chosen
or drafted tokens with the entropy and the likeliest alternatives (logp); a training step that weighs them takes the
same forward and its gradient (logp_bwd).

`run` computes an operator in elementary torch operations, or through the package's entry points where `own` is true.  A
serving loop keeps the buffers of its step's outputs, as its captured graph needs; a training step allocates them.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
PAGE = 64          # tokens of a cache page
EPS = 1e-6
THETA = 1e6        # base of the rotation's frequencies
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------ cases

def listed():
    return [
        # single tokens of 96 requests into their pages (Qwen3-4B-shaped heads)
        dict(name="append8_tokens", kind="append8", seqs=96, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=8000, Hq=32, Hkv=8, d=128,
             rot=128, inter=False),
        # a long prompt chunk and shorter ones behind it
        dict(name="append8_chunks", kind="append8", seqs=7, new_lo=500, new_hi=8000, ctx_lo=0, ctx_hi=9000, Hq=32, Hkv=8,
             d=128, rot=128, inter=False),
        # one user's next token over a long context
        dict(name="attn8_one", kind="attention8", seqs=1, new_lo=1, new_hi=1, ctx_lo=32000, ctx_hi=32000, Hq=32, Hkv=8,
             d=128),
        # single-token decode of a batch with spread contexts
        dict(name="attn8_tokens", kind="attention8", seqs=96, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=12000, Hq=32, Hkv=8,
             d=128),
        # five drafted tokens for a few long requests
        dict(name="attn8_draft", kind="attention8", seqs=6, new_lo=5, new_hi=5, ctx_lo=20000, ctx_hi=32000, Hq=32, Hkv=8,
             d=128),
        # prompt chunks and single tokens in one step, no shared heads
        dict(name="attn8_mixed", kind="attention8", seqs=13, new_lo=1, new_hi=1500, ctx_lo=0, ctx_hi=9000, Hq=24, Hkv=24,
             d=64),
        # a chunk late in a 32768-token prompt
        dict(name="attn8_prompt", kind="attention8", seqs=1, new_lo=4096, new_hi=4096, ctx_lo=28000, ctx_hi=28000, Hq=32,
             Hkv=8, d=128),
        # a decode step's sampled tokens with five alternatives each, a small odd vocabulary
        dict(name="logp_step", kind="logp", rows=24, V=32003, bf16=False, topk=5),
        # drafted tokens of a full batch, a large vocabulary
        dict(name="logp_batch", kind="logp", rows=640, V=151936, bf16=True, topk=20),
        # a training step's tokens
        dict(name="logp_train", kind="logp", rows=8192, V=151936, bf16=True, topk=0),
        # the gradient of a short odd batch
        dict(name="logp_bwd_odd", kind="logp_bwd", rows=777, V=32003, bf16=False),
        # the gradient of the training step
        dict(name="logp_bwd_train", kind="logp_bwd", rows=8192, V=151936, bf16=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["append8", "attention8", "attention8", "logp", "logp_bwd"])
    if kind in ("logp", "logp_bwd"):
        V = _log(rng, 500, 152000)
        case = dict(kind=kind, rows=_log(rng, 1, min(8192, 8192 * 152000 // (2 * V))), V=V, bf16=rng.random() < 0.5)
        return dict(case, topk=min(V, rng.choice([0, 1, rng.randint(2, 32)]))) if kind == "logp" else case
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 4, 8] if Hkv <= 4 else [1, 2, 4])
    if kind == "append8":
        one = rng.random() < 0.5
        n = _log(rng, 1, 300 if one else 12)
        hi = 1 if one else _log(rng, 2, 4000)
        return dict(kind=kind, seqs=n, new_lo=1, new_hi=hi, ctx_lo=0, ctx_hi=_log(rng, 64, 8000), Hq=Hq, Hkv=Hkv, d=d,
                    rot=rng.choice([d, d, d // 2, 16]), inter=rng.random() < 0.5)
    form = rng.choice(["tokens", "few", "chunks", "one"])
    n, lo, hi, ctx = {"tokens": (_log(rng, 1, 96), 1, 1, _log(rng, 64, 16000)),
                      "few": (_log(rng, 1, 24), 2, rng.randint(3, 17), _log(rng, 64, 30000)),
                      "chunks": (_log(rng, 2, 13), 0, _log(rng, 16, 1500), _log(rng, 64, 9000)),
                      "one": (1, 300, _log(rng, 301, 4000), _log(rng, 64, 20000))}[form]
    return dict(kind=kind, seqs=n, new_lo=lo, new_hi=hi, ctx_lo={"chunks": 0, "one": ctx}.get(form, ctx // 8), ctx_hi=ctx,
                Hq=Hq, Hkv=Hkv, d=d)


def lengths(case):
    """(cached, new) tokens of each request: fixed by the case, spread over the logarithm of its ranges."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    spread = lambda lo, hi: lo if lo == hi else max(lo, min(hi, _log(rng, lo + 1, hi + 1) - 1))  # noqa: E731
    cached = [spread(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    new = [spread(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    return cached, new if sum(new) else new[:-1] + [1]


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(shape, g, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(torch.bfloat16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tables(max_pos, rot):
    inv = THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    ang = torch.arange(max_pos, dtype=torch.float64, device=DEV)[:, None] * inv
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def _pages(total, g):
    """Block table of requests that hold `total` tokens each, over shuffled pages, and the number of pages."""
    need = [-(-n // PAGE) for n in total]
    P = sum(need) + 2
    perm = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(total), max(max(need), 1)), -1, dtype=torch.int32, device=DEV)
    have = torch.arange(table.shape[1], device=DEV) < torch.tensor(need, device=DEV)[:, None]
    table[have] = perm[:sum(need)]
    return table, P


def _norm_weight(d, g):
    return (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)


def _needed(amax):
    """The least power of two s with amax <= 448 s (448 = 0.875 * 2^9, the largest e4m3 number)."""
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -64).clamp(-64, 120)
    return torch.ldexp(torch.ones_like(amax), e)


def _cache(P, Hkv, d, g):
    """Pages of keys or values as earlier steps left them, of heads and pages of different size: numbers and scales."""
    x = torch.randn(P, Hkv, PAGE, d, generator=g, device=DEV)
    x *= torch.exp2(1.5 * torch.rand(P, Hkv, 1, 1, generator=g, device=DEV) - 0.75)
    s = _needed(x.abs().amax((2, 3)))
    return (x / s[..., None, None]).to(E4M3), s


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = dict(case)
    if kind == "append8":
        cached, new = lengths(case)
        T, H = sum(new), case["Hq"] + 2 * case["Hkv"]
        table, _ = _pages([c + n for c, n in zip(cached, new)], g)
        n, c = _ints(new), _ints(cached)
        of = torch.repeat_interleave(torch.arange(len(new), device=DEV), n.long())
        pos = torch.arange(T, device=DEV) - (n.cumsum(0) - n)[of] + c[of]
        # pages that this step does not touch are left out of the cache
        slots = (table[of, pos // PAGE].long() * PAGE + pos % PAGE).contiguous()
        touched, index = torch.unique(slots // PAGE, return_inverse=True)
        slots = (index * PAGE + slots % PAGE).contiguous()
        cos, sin = _tables(int(pos.max()) + 1, case["rot"])
        P = touched.numel()
        s.update(qkv=_normal((T, H, case["d"]), g, 1.7), wq=_norm_weight(case["d"], g), wk=_norm_weight(case["d"], g),
                 cos=cos, sin=sin, positions=pos.to(torch.int32), slots=slots)
        s["K_cache"], s["K_scale"] = _cache(P, case["Hkv"], case["d"], g)
        s["V_cache"], s["V_scale"] = _cache(P, case["Hkv"], case["d"], g)
        if own:
            from paper_2609_13141_gb300 import sas
            s["chunk"] = sas.SasChunk(len(new), case["Hq"], case["Hkv"], case["d"], table.shape[1], P, T)
            s["out"] = torch.empty(T, case["Hq"], case["d"], dtype=torch.bfloat16, device=DEV)
    elif kind == "attention8":
        cached, new = lengths(case)
        total = [c + n for c, n in zip(cached, new)]
        table, P = _pages(total, g)
        n = _ints(new)
        cu = torch.zeros(len(new) + 1, dtype=torch.int32, device=DEV)
        cu[1:] = n.cumsum(0)
        T, d = sum(new), case["d"]
        s.update(Q=_normal((T, case["Hq"], d), g, 1.5), table=table, cu=cu, kv_lens=_ints(total), n_max=max(new))
        s["K_cache"], s["K_scale"] = _cache(P, case["Hkv"], d, g)
        s["V_cache"], s["V_scale"] = _cache(P, case["Hkv"], d, g)
        if own:
            from paper_2609_13141_gb300 import sas
            s["chunk"] = sas.SasChunk(len(new), case["Hq"], case["Hkv"], d, table.shape[1], P, T)
            s["out"] = torch.empty_like(s["Q"]), torch.empty(T, case["Hq"], device=DEV)
    else:
        T, V = case["rows"], case["V"]
        dtype = torch.bfloat16 if case["bf16"] else torch.float32
        # a model's logits: a few likely tokens over a long tail, rows of different sharpness
        z = torch.empty(T, V, device=DEV).normal_(0, 1, generator=g)
        z *= 1.5 + 2 * torch.rand(T, 1, generator=g, device=DEV)
        s["logits"] = z.to(dtype)
        # sampled from the model
        z = z.sub_(torch.empty_like(z).exponential_(1, generator=g).log_())
        s["tokens"] = z.argmax(-1).to(torch.int32)
        del z
        if kind == "logp_bwd" or not case["topk"]:   # a training batch has positions that do not count
            s["tokens"][torch.rand(T, generator=g, device=DEV) < 0.05] = -1
        if kind == "logp_bwd":
            s["lse"], s["entropy"] = _row_stats(s["logits"], s["tokens"])
            s["dlogprob"] = torch.randn(T, generator=g, device=DEV)
            s["dentropy"] = 0.01 * torch.randn(T, generator=g, device=DEV)
        if own:
            from paper_2609_13141_gb300 import sas
            if kind == "logp" and case["topk"]:
                s["chunk"] = sas.SasChunk(1, 1, 1, 64, 1, 1, T)
                s["out"] = s["chunk"].logprob_buffers(T, case["topk"], DEV)
            else:
                s["layer"] = sas.SasLayer(1, 1, T, 64, 0)
    return s


# ------------------------------------------------------------------ plain forms

def _rotate(z, cos, sin, inter):
    R = 2 * cos.shape[-1]
    if inter:
        a, b = z[..., 0:R:2], z[..., 1:R:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = z[..., :R // 2], z[..., R // 2:R]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, z[..., R:]), -1)


def _norm_rope(x, w, cos, sin, inter):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return _rotate(x * r * w.float(), cos, sin, inter)


def _quantise(y, page, row, cache, scale):
    """The rows y [T, Hkv, d] into their pages.  A page whose row 0 is new starts a scale; otherwise its scale only grows,
    and rows that stay are rounded again under the larger one."""
    P, Hkv = scale.shape
    amax = torch.zeros_like(scale).scatter_reduce(0, page[:, None].expand(-1, Hkv), y.abs().amax(-1), "amax")
    fresh = torch.zeros(P, dtype=torch.bool, device=DEV).index_fill(0, page[row == 0], True)[:, None]
    s = torch.where(fresh, _needed(amax), torch.maximum(scale, _needed(amax)))
    grown = (s > scale) & ~fresh
    kept = (cache.float() * (scale / s)[..., None, None]).to(E4M3).view(torch.uint8)
    data = cache.view(torch.uint8)
    data.copy_(torch.where(grown[..., None, None], kept, data))
    data[page, :, row] = (y / s[page][..., None]).to(E4M3).view(torch.uint8)
    scale.copy_(s)


def _append8(s):
    Hq, Hkv, inter = s["Hq"], s["Hkv"], s["inter"]
    p = s["positions"].long()
    cos, sin = s["cos"][p][:, None], s["sin"][p][:, None]
    q, k, v = s["qkv"].split([Hq, Hkv, Hkv], 1)
    page, row = s["slots"] // PAGE, s["slots"] % PAGE
    _quantise(_norm_rope(k, s["wk"], cos, sin, inter), page, row, s["K_cache"], s["K_scale"])
    _quantise(v.float(), page, row, s["V_cache"], s["V_scale"])
    return dict(Q=_norm_rope(q, s["wq"], cos, sin, inter).to(torch.bfloat16), K_cache=s["K_cache"], V_cache=s["V_cache"],
                K_scale=s["K_scale"], V_scale=s["V_scale"])


def _attention8(s):
    Hkv, d, nm = s["Hkv"], s["d"], s["n_max"]
    G, cu, L = s["Hq"] // Hkv, s["cu"].long(), s["kv_lens"].long()
    n, B, T = cu[1:] - cu[:-1], s["kv_lens"].numel(), s["Q"].shape[0]
    i = torch.arange(nm, device=DEV)
    at = s["table"].clamp(min=0).long()
    held = lambda cache, scale: (cache.view(torch.uint8)[at].view(E4M3).float() * scale[at][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)  # noqa: E731,E501
    keys, vals = held(s["K_cache"], s["K_scale"]), held(s["V_cache"], s["V_scale"])
    q = s["Q"][(cu[:-1, None] + i).clamp(max=T - 1)].float().reshape(B, nm, Hkv, G, d).permute(0, 2, 3, 1, 4)
    z = (q.reshape(B, Hkv, G * nm, d) @ keys.transpose(2, 3)).reshape(B, Hkv, G, nm, -1)
    pos = (L - n)[:, None] + i
    late = torch.arange(z.shape[-1], device=DEV) > pos[..., None]
    z.mul_(1 / math.sqrt(d)).masked_fill_(late[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    e = z.sub_(m).exp_()
    l = e.sum(-1, keepdim=True)
    o = (e.reshape(B, Hkv, G * nm, -1) @ vals).reshape(B, Hkv, G, nm, d) / l
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True)
    of = (b, slice(None), slice(None), t - cu[b])
    return dict(O=o[of].reshape(T, -1, d).to(torch.bfloat16), LSE=(m + l.log())[..., 0][of].reshape(T, -1))


def _row_stats(logits, tokens):
    """log sum exp and entropy of each row that counts, 0 for the others."""
    z = logits.float()
    m = z.amax(-1, keepdim=True)
    z = z.sub_(m) if z.data_ptr() != logits.data_ptr() else z - m
    e = z.exp()
    l = e.sum(-1)
    h = l.log() - e.mul_(z).sum(-1) / l
    counts = tokens >= 0
    return torch.where(counts, m[:, 0] + l.log(), 0), torch.where(counts, h, 0)


def _logp(s):
    lse, entropy = _row_stats(s["logits"], s["tokens"])
    counts = s["tokens"] >= 0
    z = s["logits"].gather(1, s["tokens"].long().clamp(min=0)[:, None])[:, 0].float()
    out = dict(logprob=torch.where(counts, z - lse, 0), entropy=entropy, lse=lse)
    if s["topk"]:
        # the likeliest, the lowest index of equal ones: order by the logit's bits, then by the index
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()   # one zero
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        index = torch.arange(s["V"], device=DEV)
        top = torch.topk(order * 2 ** 32 + (2 ** 32 - 1 - index), s["topk"]).values
        idx = 2 ** 32 - 1 - torch.remainder(top, 2 ** 32)
        out.update(top_index=idx.int(), top_logprob=s["logits"].gather(1, idx).float() - lse[:, None])
    return out


def _logp_bwd(s):
    counts = s["tokens"] >= 0
    logp = s["logits"].float() - s["lse"][:, None]
    p = logp.exp()
    g = logp.add_(s["entropy"][:, None]).mul_(s["dentropy"][:, None]).add_(s["dlogprob"][:, None]).mul_(p).neg_()
    t = s["tokens"].long().clamp(min=0)[:, None]
    g.scatter_add_(1, t, s["dlogprob"][:, None])
    g.masked_fill_(~counts[:, None], 0)
    return dict(dlogits=g.to(s["logits"].dtype))


PLAIN = dict(append8=_append8, attention8=_attention8, logp=_logp, logp_bwd=_logp_bwd)


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["kind"]
    if not own:
        return PLAIN[kind](s)
    if kind == "append8":
        Q = s["chunk"].append8(s["qkv"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], s["slots"], s["K_cache"],
                               s["V_cache"], s["K_scale"], s["V_scale"], eps=EPS, interleaved=s["inter"], out=s["out"])
        return dict(Q=Q, K_cache=s["K_cache"], V_cache=s["V_cache"], K_scale=s["K_scale"], V_scale=s["V_scale"])
    if kind == "attention8":
        O, LSE = s["chunk"].attention8(s["Q"], s["K_cache"], s["V_cache"], s["K_scale"], s["V_scale"], s["table"], s["cu"],
                                       s["kv_lens"], out=s["out"])
        return dict(O=O, LSE=LSE)
    if kind == "logp_bwd":
        return dict(dlogits=s["layer"].token_logprobs_bwd(s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogprob"],
                                                          s["dentropy"]))
    if s["topk"]:
        r = s["chunk"].logprobs(s["logits"], s["tokens"], s["topk"], out=s["out"])
        return dict(logprob=r.logprob, entropy=r.entropy, lse=r.lse, top_index=r.top_index, top_logprob=r.top_logprob)
    r = s["layer"].token_logprobs(s["logits"], s["tokens"])
    return dict(logprob=r.logprob, entropy=r.entropy, lse=r.lse)


# ------------------------------------------------------------------ work and 64-bit values

def work(case):
    kind = case["kind"]
    if kind in ("logp", "logp_bwd"):
        T, n = case["rows"], case["rows"] * case["V"]
        size = n * (2 if case["bf16"] else 4)
        if kind == "logp":
            return dict(bytes=size + T * (16 + 8 * case["topk"]), flops=5 * n)
        return dict(bytes=2 * size + 20 * T, flops=6 * n)
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    cached, new = lengths(case)
    T = sum(new)
    if kind == "append8":
        # the projection's rows, the queries in bf16, keys and values in 8 bits, the pages' scales
        pages = sum(-(-(c + n) // PAGE) - c // PAGE for c, n in zip(cached, new) if n)
        return dict(bytes=T * ((Hq + 2 * Hkv) * d * 2 + Hq * d * 2 + 2 * Hkv * d + 12 + 4 * case["rot"]) + pages * Hkv * 16,
                    flops=T * (Hq + Hkv) * d * 8 + T * Hkv * d * 4)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, new))
    held = sum(c + n for c, n in zip(cached, new) if n)
    return dict(bytes=held * Hkv * 2 * d + held // PAGE * Hkv * 8 + T * Hq * (4 * d + 4), flops=4 * d * Hq * pairs)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "append8":
        return _exact_append8(s)
    if kind == "attention8":
        return _exact_attention8(s)
    rows, V = s["tokens"].tolist(), case["V"]
    f64 = dict(dtype=torch.float64, device=DEV)
    if kind == "logp_bwd":
        out = torch.zeros(len(rows), V, **f64)
        for t0 in range(0, len(rows), 1024):
            at = slice(t0, t0 + 1024)
            logp = torch.log_softmax(s["logits"][at].double(), -1)
            p = logp.exp()
            h = -(p * logp).sum(-1, keepdim=True)
            hit = torch.arange(V, device=DEV) == s["tokens"][at, None]
            d = s["dlogprob"][at, None] * (hit.double() - p) - s["dentropy"][at, None] * p * (logp + h)
            out[at] = torch.where(s["tokens"][at, None] >= 0, d, 0)
        return dict(dlogits=out)
    out = {k: torch.zeros(len(rows), **f64) for k in ("logprob", "entropy", "lse")}
    if case["topk"]:
        out.update(top_index=torch.empty(len(rows), case["topk"], dtype=torch.int32, device=DEV),
                   top_logprob=torch.empty(len(rows), case["topk"], **f64))
    for t, x in enumerate(rows):
        if x < 0:
            continue
        z = s["logits"][t].double()
        out["lse"][t] = lse = torch.logsumexp(z, 0)
        logp = z - lse
        out["logprob"][t] = logp[x]
        out["entropy"][t] = -(logp.exp() * logp).sum()
        if case["topk"]:
            order = torch.sort(z, descending=True, stable=True).indices[:case["topk"]]
            out["top_index"][t] = order.int()
            out["top_logprob"][t] = logp[order]
    return out


def _exact_append8(s):
    """Values before their rounding to 8 bits, in units of the page's scale."""
    Hq, Hkv, rot, inter = s["Hq"], s["Hkv"], s["rot"], s["inter"]
    p = s["positions"].long()
    phase = torch.complex(s["cos"].double(), s["sin"].double())[p][:, None]

    def turned(x, w):
        x = x.double()
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
        y = x[..., :rot]
        pair = y.unflatten(-1, (rot // 2, 2)) if inter else y.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * phase)
        y = pair.flatten(-2) if inter else pair.transpose(-1, -2).flatten(-2)
        return torch.cat((y, x[..., rot:]), -1)

    out = dict(Q=turned(s["qkv"][:, :Hq], s["wq"]))
    new = dict(K=turned(s["qkv"][:, Hq:Hq + Hkv], s["wk"]), V=s["qkv"][:, Hq + Hkv:].double())
    slots = s["slots"].tolist()
    pages = {}
    for t, slot in enumerate(slots):
        pages.setdefault(slot // PAGE, []).append((t, slot % PAGE))
    for name in ("K", "V"):
        cache, scale = s[name + "_cache"].double(), s[name + "_scale"].double()
        for page, rows in pages.items():
            ts, rs = [t for t, _ in rows], [r for _, r in rows]
            y = new[name][ts]                                        # [n, Hkv, d]
            m, e = torch.frexp(y.abs().amax((0, 2)) / 448)           # a power of two has m = 0.5
            need = torch.exp2((e - (m == 0.5).int()).clamp(-64, 120).double())
            if 0 not in rs:
                need = torch.maximum(scale[page], need)
                cache[page] *= (scale[page] / need)[:, None, None]
            cache[page][:, rs] = (y / need[:, None]).transpose(0, 1)
            scale[page] = need
        out.update({name + "_cache": cache, name + "_scale": scale})
    return out


def _exact_attention8(s):
    Hkv, d = s["Hkv"], s["d"]
    G, T = s["Hq"] // Hkv, s["Q"].shape[0]
    O = torch.empty(T, s["Hq"], d, dtype=torch.float64, device=DEV)
    LSE = torch.empty(T, s["Hq"], dtype=torch.float64, device=DEV)
    cu, total = s["cu"].tolist(), s["kv_lens"].tolist()

    def held(name, pages, g, L):
        x = s[name + "_cache"].view(torch.uint8)[pages, g].view(E4M3).double() * s[name + "_scale"][pages, g].double()[:, None, None]
        return x.reshape(-1, d)[:L]

    for b, L in enumerate(total):
        pages = s["table"][b, :-(-L // PAGE)].long()
        for g in range(Hkv):
            K, V = held("K", pages, g, L), held("V", pages, g, L)
            for t0 in range(cu[b], cu[b + 1], 512):
                t1 = min(t0 + 512, cu[b + 1])
                pos = torch.arange(t0, t1, device=DEV) - cu[b + 1] + L
                z = torch.einsum("tgd,ld->tgl", s["Q"][t0:t1, g * G:(g + 1) * G].double(), K) / math.sqrt(d)
                z.masked_fill_((torch.arange(L, device=DEV) > pos[:, None])[:, None], -math.inf)
                LSE[t0:t1, g * G:(g + 1) * G] = lse = torch.logsumexp(z, -1)
                O[t0:t1, g * G:(g + 1) * G] = torch.einsum("tgl,ld->tgd", (z - lse[..., None]).exp(), V)
    return dict(O=O, LSE=LSE)
