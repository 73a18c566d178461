"""Timed cases of the serving-step and projection operators.

One step of serving over the paged cache is: page assignment and slot map (plan), per-head norm + rotation + cache append
(append), attention of the new tokens over the cache (attention), verification of drafted tokens (verify).  Training
takes the same norm + rotation between the QKV projection and the attention (rope_fwd, rope_bwd).

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


# ------------------------------------------------------------------ cases

def listed():
    return [
        # one decode step of 256 requests: every length grows by one, every 64th opens a page
        dict(name="plan_decode", kind="plan", seqs=256, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=32000, max_blocks=512),
        # admission of many prompts at once, some requests idle
        dict(name="plan_prompts", kind="plan", seqs=1500, new_lo=0, new_hi=1900, ctx_lo=0, ctx_hi=7000, max_blocks=512),
        # single tokens of 96 requests into their pages (Qwen3-4B-shaped heads)
        dict(name="append_tokens", kind="append", seqs=96, new_lo=1, new_hi=1, ctx_lo=1, ctx_hi=8000, Hq=32, Hkv=8, d=128,
             rot=128, inter=False),
        # a 16K-token prompt chunk and shorter ones behind it
        dict(name="append_chunks", kind="append", seqs=7, new_lo=500, new_hi=8000, ctx_lo=0, ctx_hi=9000, Hq=32, Hkv=8,
             d=128, rot=128, inter=False),
        # training prologue of an odd-length batch, no shared heads, partial interleaved rotation
        dict(name="rope_fwd_odd", kind="rope_fwd", B=2, N=4549, Hq=24, Hkv=24, d=64, rot=32, inter=True),
        # its gradient at the 32768-token training length
        dict(name="rope_bwd_32k", kind="rope_bwd", B=1, N=32768, Hq=32, Hkv=8, d=128, rot=128, inter=False),
        # single-token decode of a batch with spread contexts
        dict(name="attn_tokens", kind="attention", seqs=96, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=12000, Hq=32, Hkv=8,
             d=128),
        # five drafted tokens for a few long requests
        dict(name="attn_draft", kind="attention", seqs=6, new_lo=5, new_hi=5, ctx_lo=20000, ctx_hi=32000, Hq=32, Hkv=8,
             d=128),
        # prompt chunks and single tokens in one step
        dict(name="attn_mixed", kind="attention", seqs=13, new_lo=1, new_hi=1500, ctx_lo=0, ctx_hi=9000, Hq=24, Hkv=24,
             d=64),
        # a chunk late in a 32768-token prompt
        dict(name="attn_prompt", kind="attention", seqs=1, new_lo=4096, new_hi=4096, ctx_lo=28000, ctx_hi=28000, Hq=32,
             Hkv=8, d=128),
        # four drafts for a handful of requests, a small odd vocabulary
        dict(name="verify_small", kind="verify", seqs=8, drafts=4, V=32003),
        # a full batch, a large vocabulary
        dict(name="verify_batch", kind="verify", seqs=128, drafts=5, V=151936),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "rope_fwd", "rope_bwd", "attention", "attention", "verify"])
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12])
    Hq = Hkv * rng.choice([1, 2, 4, 8] if Hkv <= 4 else [1, 2, 4])
    rot = rng.choice([d, d, d // 2, 16])
    if kind == "plan":
        n = _log(rng, 1, 1500)
        hi = 1 if rng.random() < 0.4 else _log(rng, 2, 1900)
        return dict(kind=kind, seqs=n, new_lo=rng.choice([0, 1]), new_hi=hi, ctx_lo=0, ctx_hi=_log(rng, 64, 30000),
                    max_blocks=512)
    if kind == "append":
        one = rng.random() < 0.5
        n = _log(rng, 1, 300 if one else 12)
        hi = 1 if one else _log(rng, 2, 4000)
        return dict(kind=kind, seqs=n, new_lo=1, new_hi=hi, ctx_lo=0, ctx_hi=_log(rng, 64, 8000), Hq=Hq, Hkv=Hkv, d=d, rot=rot,
                    inter=rng.random() < 0.5)
    if kind in ("rope_fwd", "rope_bwd"):
        B = rng.choice([1, 2, 3])
        longest = min(32768, 32768 * 48 * 128 // (B * (Hq + 2 * Hkv) * d))
        return dict(kind=kind, B=B, N=_log(rng, 33, longest), Hq=Hq, Hkv=Hkv, d=d, rot=rot, inter=rng.random() < 0.5)
    if kind == "attention":
        form = rng.choice(["tokens", "few", "chunks", "one"])
        n, lo, hi, ctx = {"tokens": (_log(rng, 1, 96), 1, 1, _log(rng, 64, 16000)),
                          "few": (_log(rng, 1, 24), 2, rng.randint(3, 17), _log(rng, 64, 30000)),
                          "chunks": (_log(rng, 2, 13), 0, _log(rng, 16, 1500), _log(rng, 64, 9000)),
                          "one": (1, 300, _log(rng, 301, 4000), _log(rng, 64, 20000))}[form]
        return dict(kind=kind, seqs=n, new_lo=lo, new_hi=hi, ctx_lo={"chunks": 0, "one": ctx}.get(form, ctx // 8),
                    ctx_hi=ctx, Hq=Hq, Hkv=Hkv, d=d)
    return dict(kind=kind, seqs=_log(rng, 1, 128), drafts=rng.randint(1, 12), V=_log(rng, 1000, 152000))


def lengths(case):
    """(cached, new) tokens of each request: fixed by the case, spread over the logarithm of its ranges."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    spread = lambda lo, hi: lo if lo == hi else max(lo, min(hi, _log(rng, lo + 1, hi + 1) - 1))  # noqa: E731
    cached = [spread(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    new = [spread(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    return cached, new if sum(new) else new[:-1] + [1]


def draft_counts(case):
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    return [case["drafts"] if rng.random() < 0.7 else rng.randint(0, case["drafts"]) for _ in range(case["seqs"])]


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


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = dict(case)
    if kind == "plan":
        cached, new = lengths(case)
        need = [-(-(c + n) // PAGE) - -(-c // PAGE) for c, n in zip(cached, new)]
        held = [-(-c // PAGE) for c in cached]
        P = sum(need) + sum(held) + 64
        perm = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
        table = torch.full((case["seqs"], case["max_blocks"]), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(case["max_blocks"], device=DEV) < torch.tensor(held, device=DEV)[:, None]] = perm[:sum(held)]
        s.update(seq_lens=_ints(cached), new_lens=_ints(new), free_pages=perm[sum(held):].contiguous(),
                 free_begin=_ints([seed % 7]), table=table, T=max(1, sum(new)), P=P)
        if own:
            from paper_2609_13141_gb300 import sas
            s["chunk"] = sas.SasChunk(case["seqs"], 1, 1, 64, case["max_blocks"], P, s["T"])
            s["out"] = s["chunk"].plan_buffers(case["seqs"], s["T"], DEV)
    elif kind == "append":
        cached, new = lengths(case)
        T, H = sum(new), case["Hq"] + 2 * case["Hkv"]
        table, P = _pages([c + n for c, n in zip(cached, new)], g)
        n, c = _ints(new), _ints(cached)
        of = torch.repeat_interleave(torch.arange(len(new), device=DEV), n.long())
        pos = torch.arange(T, device=DEV) - (n.cumsum(0) - n)[of] + c[of]
        # pages that this step does not touch are left out of the cache
        slots = (table[of, pos // PAGE].long() * PAGE + pos % PAGE).contiguous()
        touched, index = torch.unique(slots // PAGE, return_inverse=True)
        slots = (index * PAGE + slots % PAGE).contiguous()
        cos, sin = _tables(int(pos.max()) + 1, case["rot"])
        s.update(qkv=_normal((T, H, case["d"]), g, 1.7), wq=_norm_weight(case["d"], g), wk=_norm_weight(case["d"], g),
                 cos=cos, sin=sin, positions=pos.to(torch.int32), slots=slots,
                 K_cache=_normal((touched.numel(), case["Hkv"], PAGE, case["d"]), g),
                 V_cache=_normal((touched.numel(), case["Hkv"], PAGE, case["d"]), g))
        if own:
            from paper_2609_13141_gb300 import sas
            s["chunk"] = sas.SasChunk(len(new), case["Hq"], case["Hkv"], case["d"], table.shape[1], touched.numel(), T)
            s["out"] = torch.empty(T, case["Hq"], case["d"], dtype=torch.bfloat16, device=DEV)
    elif kind in ("rope_fwd", "rope_bwd"):
        B, N, Hq, Hkv, d = (case[k] for k in ("B", "N", "Hq", "Hkv", "d"))
        cos, sin = _tables(N, case["rot"])
        s.update(qkv=_normal((B, N, Hq + 2 * Hkv, d), g, 1.7), wq=_norm_weight(d, g), wk=_norm_weight(d, g), cos=cos, sin=sin)
        if kind == "rope_bwd":
            s.update(dQ=_normal((B, Hq, N, d), g, 0.3), dK=_normal((B, Hkv, N, d), g, 0.3),
                     dV=_normal((B, Hkv, N, d), g, 0.3))
        if own:
            from paper_2609_13141_gb300 import sas
            s["layer"] = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    elif kind == "attention":
        cached, new = lengths(case)
        total = [c + n for c, n in zip(cached, new)]
        table, P = _pages(total, g)
        n = _ints(new)
        cu = torch.zeros(len(new) + 1, dtype=torch.int32, device=DEV)
        cu[1:] = n.cumsum(0)
        T, d = sum(new), case["d"]
        s.update(Q=_normal((T, case["Hq"], d), g, 1.5), K_cache=_normal((P, case["Hkv"], PAGE, d), g),
                 V_cache=_normal((P, case["Hkv"], PAGE, d), g), table=table, cu=cu, kv_lens=_ints(total),
                 n_max=max(new))
        if own:
            from paper_2609_13141_gb300 import sas
            s["chunk"] = sas.SasChunk(len(new), case["Hq"], case["Hkv"], d, table.shape[1], P, T)
            s["out"] = torch.empty_like(s["Q"]), torch.empty(T, case["Hq"], device=DEV)
    else:
        counts, V = draft_counts(case), case["V"]
        B, Td = case["seqs"], sum(counts)
        cu = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
        cu[1:] = _ints(counts).cumsum(0)
        # target and draft distributions of a model: a few likely tokens over a long tail, the draft near the target
        target = torch.empty(Td + B, V, device=DEV).normal_(0, 2.5, generator=g)
        last = torch.zeros(Td + B, dtype=torch.bool, device=DEV)
        last[cu[1:].long() + torch.arange(B, device=DEV)] = True
        draft = target[~last]
        draft = torch.softmax(draft + 0.7 * torch.empty_like(draft).normal_(0, 1, generator=g), -1)
        target = torch.softmax(target, -1)
        race = torch.empty_like(draft).exponential_(1, generator=g)
        tokens = (draft / race).argmax(-1).to(torch.int32) if Td else torch.zeros(0, dtype=torch.int32, device=DEV)
        del race
        s.update(cu=cu, target=target, draft=draft, tokens=tokens, u=torch.rand(Td, generator=g, device=DEV),
                 noise=torch.empty(B, V, device=DEV).exponential_(1, generator=g).clamp_min_(1e-30))
        if own:
            from paper_2609_13141_gb300 import sas
            s["chunk"] = sas.SasChunk(B, 1, 1, 64, 1, 1, max(1, Td))
            s["out"] = _ints([0] * B), _ints([[0] * (case["drafts"] + 1)] * B)
    return s


# ------------------------------------------------------------------ plain forms

def _plan(s):
    c, n, T, F = s["seq_lens"].long(), s["new_lens"].long(), s["T"], s["free_pages"].numel()
    have, tot = (c + PAGE - 1) // PAGE, (c + n + PAGE - 1) // PAGE
    need = tot - have
    begin = s["free_begin"].long()[0]
    fits = (need.sum() <= F - begin) & (n.sum() <= T) & (n >= 0).all() & (c >= 0).all() & (tot <= s["max_blocks"]).all()
    n, tot, need = n * fits, torch.where(fits, tot, have), need * fits
    off = need.cumsum(0) - need
    m = torch.arange(s["max_blocks"], device=DEV)
    fresh = (m >= have[:, None]) & (m < tot[:, None])
    page = s["free_pages"][(begin + off[:, None] + m - have[:, None]).clamp(0, F - 1)]
    s["table"].copy_(torch.where(fresh, page, s["table"]))
    cu = torch.zeros(n.numel() + 1, dtype=torch.int64, device=DEV)
    cu[1:] = n.cumsum(0)
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=n.numel() - 1)
    live = t < cu[-1]
    pos = torch.where(live, c[b] + t - cu[b], -1)
    slot = s["table"][b, pos.clamp(min=0) // PAGE].long() * PAGE + pos % PAGE
    return dict(kv_lens=(c + n).int(), cu=cu.int(), positions=pos.int(), slots=torch.where(live, slot, -1),
                free_end=(begin + need.sum()).int().reshape(1), table=s["table"])


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
    return _rotate(x * r * w.float(), cos, sin, inter).to(torch.bfloat16)


def _norm_rope_grad(x, w, cos, sin, inter, dy):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh = x * r
    dz = _rotate(dy.float(), cos, -sin, inter)
    u = dz * w.float()
    dx = r * (u - xh * (u * xh).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), (dz * xh).sum((0, 1, 2))


def _append(s):
    Hq, Hkv, inter = s["Hq"], s["Hkv"], s["inter"]
    p = s["positions"].long()
    cos, sin = s["cos"][p][:, None], s["sin"][p][:, None]
    q, k, v = s["qkv"].split([Hq, Hkv, Hkv], 1)
    page, row = s["slots"] // PAGE, s["slots"] % PAGE
    s["K_cache"][page, :, row] = _norm_rope(k, s["wk"], cos, sin, inter)
    s["V_cache"][page, :, row] = v
    return dict(Q=_norm_rope(q, s["wq"], cos, sin, inter), K_cache=s["K_cache"], V_cache=s["V_cache"])


def _rope_fwd(s):
    q, k, v = s["qkv"].split([s["Hq"], s["Hkv"], s["Hkv"]], 2)
    cos, sin = s["cos"][:s["N"], None], s["sin"][:s["N"], None]
    bhnd = lambda x: x.transpose(1, 2).contiguous()  # noqa: E731
    return dict(Q=bhnd(_norm_rope(q, s["wq"], cos, sin, s["inter"])), K=bhnd(_norm_rope(k, s["wk"], cos, sin, s["inter"])),
                V=bhnd(v))


def _rope_bwd(s):
    q, k, _ = s["qkv"].split([s["Hq"], s["Hkv"], s["Hkv"]], 2)
    cos, sin = s["cos"][:s["N"], None], s["sin"][:s["N"], None]
    dq, dwq = _norm_rope_grad(q, s["wq"], cos, sin, s["inter"], s["dQ"].transpose(1, 2))
    dk, dwk = _norm_rope_grad(k, s["wk"], cos, sin, s["inter"], s["dK"].transpose(1, 2))
    return dict(dqkv=torch.cat((dq, dk, s["dV"].transpose(1, 2)), 2), dwq=dwq, dwk=dwk)


def _attention(s):
    Hkv, d, nm = s["Hkv"], s["d"], s["n_max"]
    G, cu, L = s["Hq"] // Hkv, s["cu"].long(), s["kv_lens"].long()
    n, B, T = cu[1:] - cu[:-1], s["kv_lens"].numel(), s["Q"].shape[0]
    i = torch.arange(nm, device=DEV)
    keys = s["K_cache"][s["table"].clamp(min=0).long()].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
    vals = s["V_cache"][s["table"].clamp(min=0).long()].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
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
    at = (b, slice(None), slice(None), t - cu[b])
    return dict(O=o[at].reshape(T, -1, d).to(torch.bfloat16), LSE=(m + l.log())[..., 0][at].reshape(T, -1))


def _verify(s):
    cu, W, V = s["cu"].long(), s["drafts"], s["V"]
    c0, n = cu[:-1], cu[1:] - cu[:-1]
    B = n.numel()
    b = torch.arange(B, device=DEV)
    j = torch.arange(W, device=DEV)
    live = j < n[:, None]
    at = (c0[:, None] + j).clamp(max=max(0, s["tokens"].numel() - 1))
    if s["tokens"].numel():
        tok = s["tokens"].long()[at]
        ok = live & (s["u"][at] * s["draft"][at, tok] < s["target"][(c0 + b)[:, None] + torch.where(live, j, 0), tok])
        drafted = torch.where(live, tok, -1)
        a = ok.long().cumprod(1).sum(1)
        q = torch.where((a == n)[:, None], 0, s["draft"][(c0 + a).clamp(max=s["tokens"].numel() - 1)])
    else:
        drafted = torch.full((B, W), -1, dtype=torch.int64, device=DEV)
        a, q = torch.zeros_like(n), torch.zeros(B, V, device=DEV)
    p = s["target"][c0 + b + a]
    w = (p - q).clamp(min=0)
    w = torch.where(w.amax(1, keepdim=True) > 0, w, p)
    score = w / s["noise"]
    best = score.amax(1, keepdim=True)
    pick = torch.where(score == best, torch.arange(V, device=DEV), V).amin(1)
    out = torch.full((B, W + 1), -1, dtype=torch.int64, device=DEV)
    out[:, :W] = torch.where(j < a[:, None], drafted, -1)
    out[b, a] = torch.where(best[:, 0] > 0, pick, -1)
    return dict(accepted=a.int(), tokens=out.int())


PLAIN = dict(plan=_plan, append=_append, rope_fwd=_rope_fwd, rope_bwd=_rope_bwd, attention=_attention, verify=_verify)


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["kind"]
    if not own:
        return PLAIN[kind](s)
    if kind == "plan":
        p = s["chunk"].plan(s["seq_lens"], s["new_lens"], s["free_pages"], s["free_begin"], s["table"], s["T"], out=s["out"])
        return dict(kv_lens=p.kv_lens, cu=p.cu_new, positions=p.positions, slots=p.slots, free_end=p.free_end,
                    table=s["table"])
    if kind == "append":
        Q = s["chunk"].append(s["qkv"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], s["slots"], s["K_cache"],
                              s["V_cache"], eps=EPS, interleaved=s["inter"], out=s["out"])
        return dict(Q=Q, K_cache=s["K_cache"], V_cache=s["V_cache"])
    if kind == "rope_fwd":
        Q, K, V = s["layer"].qk_norm_rope(s["qkv"], s["wq"], s["wk"], s["cos"], s["sin"], eps=EPS, interleaved=s["inter"])
        return dict(Q=Q, K=K, V=V)
    if kind == "rope_bwd":
        dqkv, dwq, dwk = s["layer"].qk_norm_rope_bwd(s["qkv"], s["wq"], s["wk"], s["cos"], s["sin"], s["dQ"], s["dK"],
                                                     s["dV"], eps=EPS, interleaved=s["inter"])
        return dict(dqkv=dqkv, dwq=dwq, dwk=dwk)
    if kind == "attention":
        O, LSE = s["chunk"].attention(s["Q"], s["K_cache"], s["V_cache"], s["table"], s["cu"], s["kv_lens"], out=s["out"])
        return dict(O=O, LSE=LSE)
    accepted, tokens = s["chunk"].verify(s["tokens"], s["cu"], s["target"], s["draft"], s["u"], s["noise"], s["drafts"],
                                         out=s["out"])
    return dict(accepted=accepted, tokens=tokens)


# ------------------------------------------------------------------ work and 64-bit values

def work(case):
    kind = case["kind"]
    if kind == "plan":
        cached, new = lengths(case)
        need = sum(-(-(c + n) // PAGE) - -(-c // PAGE) for c, n in zip(cached, new))
        return dict(bytes=16 * case["seqs"] + 12 * sum(new) + 8 * need, flops=0)
    if kind == "verify":
        counts = draft_counts(case)
        # the first rejected row of p and q and the noise row of each request
        return dict(bytes=case["seqs"] * case["V"] * 12 + 16 * sum(counts), flops=2 * case["seqs"] * case["V"])
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    row = (Hq + 2 * Hkv) * d * 2
    if kind == "append":
        _, new = lengths(case)
        return dict(bytes=sum(new) * (2 * row + 12 + 4 * case["rot"]), flops=sum(new) * (Hq + Hkv) * d * 8)
    if kind in ("rope_fwd", "rope_bwd"):
        T = case["B"] * case["N"]
        if kind == "rope_fwd":
            return dict(bytes=T * 2 * row + case["N"] * 4 * case["rot"], flops=T * (Hq + Hkv) * d * 8)
        return dict(bytes=T * (2 * row + (Hq + Hkv) * d * 2) + case["N"] * 4 * case["rot"], flops=T * (Hq + Hkv) * d * 18)
    cached, new = lengths(case)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, new))
    held = sum(c + n for c, n in zip(cached, new) if n)
    return dict(bytes=held * Hkv * d * 4 + sum(new) * Hq * (4 * d + 4), flops=4 * d * Hq * pairs)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "plan":
        return _exact_plan(s)
    if kind == "verify":
        return _exact_verify(s)
    if kind == "attention":
        return _exact_attention(s)
    Hq, Hkv, rot, inter = case["Hq"], case["Hkv"], case["rot"], case["inter"]

    def turned(x, w, phase):
        """Norm, weight, then a product with exp(i angle) on the rotated pairs."""
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        y = x[..., :rot]
        pair = y.unflatten(-1, (rot // 2, 2)) if inter else y.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * phase)
        y = pair.flatten(-2) if inter else pair.transpose(-1, -2).flatten(-2)
        return torch.cat((y, x[..., rot:]), -1)

    qkv = s["qkv"].double()
    wq, wk = s["wq"].double(), s["wk"].double()
    phase = torch.complex(s["cos"].double(), s["sin"].double())
    if kind == "append":
        phase = phase[s["positions"].long()][:, None]
        K, V = s["K_cache"].double(), s["V_cache"].double()
        at = (s["slots"] // PAGE, slice(None), s["slots"] % PAGE)
        K[at], V[at] = turned(qkv[:, Hq:Hq + Hkv], wk, phase), qkv[:, Hq + Hkv:]
        return dict(Q=turned(qkv[:, :Hq], wq, phase), K_cache=K, V_cache=V)
    phase = phase[:case["N"]][None, :, None]
    if kind == "rope_fwd":
        q, k = turned(qkv[:, :, :Hq], wq, phase), turned(qkv[:, :, Hq:Hq + Hkv], wk, phase)
        return dict(Q=q.transpose(1, 2).contiguous(), K=k.transpose(1, 2).contiguous(),
                    V=qkv[:, :, Hq + Hkv:].transpose(1, 2).contiguous())
    grads, dws = [], []
    for part, w, dy in ((qkv[:, :, :Hq], wq, s["dQ"]), (qkv[:, :, Hq:Hq + Hkv], wk, s["dK"])):
        part, w = part.clone().requires_grad_(), w.clone().requires_grad_()
        turned(part, w, phase).backward(dy.double().transpose(1, 2))
        grads.append(part.grad)
        dws.append(w.grad)
    return dict(dqkv=torch.cat(grads + [s["dV"].double().transpose(1, 2)], 2), dwq=dws[0], dwk=dws[1])


def _exact_plan(s):
    cached, new, free = s["seq_lens"].tolist(), s["new_lens"].tolist(), s["free_pages"].tolist()
    table, at = s["table"].tolist(), int(s["free_begin"])
    cu, positions, slots = [0], [], []
    for b, (c, n) in enumerate(zip(cached, new)):
        for p in range(c, c + n):
            if p % PAGE == 0:
                table[b][p // PAGE] = free[at]
                at += 1
            positions.append(p)
            slots.append(table[b][p // PAGE] * PAGE + p % PAGE)
        cu.append(cu[-1] + n)
    pad = [-1] * (s["T"] - len(slots))
    return dict(kv_lens=_ints([c + n for c, n in zip(cached, new)]), cu=_ints(cu), positions=_ints(positions + pad),
                slots=torch.tensor(slots + pad, device=DEV), free_end=_ints([at]), table=_ints(table))


def _exact_attention(s):
    Hkv, d = s["Hkv"], s["d"]
    G, T = s["Hq"] // Hkv, s["Q"].shape[0]
    O = torch.empty(T, s["Hq"], d, dtype=torch.float64, device=DEV)
    LSE = torch.empty(T, s["Hq"], dtype=torch.float64, device=DEV)
    cu, total = s["cu"].tolist(), s["kv_lens"].tolist()
    for b, L in enumerate(total):
        pages = s["table"][b, :-(-L // PAGE)].long()
        for g in range(Hkv):
            K = s["K_cache"][pages, g].reshape(-1, d)[:L].double()
            V = s["V_cache"][pages, g].reshape(-1, d)[:L].double()
            for t0 in range(cu[b], cu[b + 1], 512):
                t1 = min(t0 + 512, cu[b + 1])
                pos = torch.arange(t0, t1, device=DEV) - cu[b + 1] + L
                z = torch.einsum("tgd,ld->tgl", s["Q"][t0:t1, g * G:(g + 1) * G].double(), K) / math.sqrt(d)
                z.masked_fill_((torch.arange(L, device=DEV) > pos[:, None])[:, None], -math.inf)
                LSE[t0:t1, g * G:(g + 1) * G] = lse = torch.logsumexp(z, -1)
                O[t0:t1, g * G:(g + 1) * G] = torch.einsum("tgl,ld->tgd", (z - lse[..., None]).exp(), V)
    return dict(O=O, LSE=LSE)


def _exact_verify(s):
    cu, accepted, tokens = s["cu"].tolist(), [], []
    for b in range(len(cu) - 1):
        row, drafted = [], s["tokens"][cu[b]:cu[b + 1]].tolist()
        res = None
        for j, x in enumerate(drafted):
            p, q = s["target"][cu[b] + b + j].double(), s["draft"][cu[b] + j].double()
            if not float(s["u"][cu[b] + j].double() * q[x]) < float(p[x]):
                res = (p - q).clamp(min=0)
                res = res if float(res.max()) > 0 else p
                break
            row.append(x)
        accepted.append(len(row))
        if res is None:
            res = s["target"][cu[b + 1] + b].double()
        row.append(int((res / s["noise"][b].double()).argmax()))
        tokens.append(row + [-1] * (s["drafts"] + 1 - len(row)))
    return dict(accepted=_ints(accepted), tokens=_ints(tokens))
