"""Steps over an 8-bit cache as a server runs them: plan, append8, attention8 and logprobs captured in one graph, replayed while
lengths, tokens and pages change."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas
from tests.test_gpu_attention8 import DEV, E4, I32, _compare

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _steps(kind):
    """New tokens of each request, and the size of the step's activations (0: zeros)."""
    rng = np.random.default_rng(3)
    if kind == "chunks":
        new = [[70, 10, 0], [1, 1, 90], [5, 2, 5], [1, 1, 1], [0, 0, 0], [1, 1, 1], [40, 1, 3], [64, 63, 1]]
        return 3, 128, list(zip(new, [1, 4, 0.5, 0, 1, 16, 1, 64]))
    new = rng.integers(0, 3, (60, 6)).tolist()
    return 6, 12, list(zip(new, (2.0 ** rng.integers(-2, 5, 60) * (rng.random(60) < 0.9)).tolist()))


@pytest.mark.parametrize("kind", ["chunks", "tokens"])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 4, 2)])
def test_captured_steps(kind, d, Hq, Hkv):
    """The cache holds every token's normed and turned key and its value to as many roundings as its page's scale has grown
    (one more than that): half a step each, 2^-4 of the number or 2^-10 of the scale; keys are off by 2^-19 of the row's largest
    before they are turned (test_gpu_append8), which is at most sqrt(2) of the largest after.  Each step's attention is that over the cache as it stands."""
    B, T, steps = _steps(kind)
    g = torch.Generator(device=DEV).manual_seed(11)
    P, W, V = 8 * B, 8, 1000
    H = Hq + 2 * Hkv
    ch = sas.SasChunk(B, Hq, Hkv, d, W, P, T)
    K8, V8 = (torch.full((P, Hkv, 64, d), 0x7F, dtype=torch.uint8, device=DEV).view(E4) for _ in range(2))
    sk, sv = (torch.full((P, Hkv), math.nan, device=DEV) for _ in range(2))
    table = torch.full((B, W), -1, dtype=I32, device=DEV)
    free, begin = torch.randperm(P, generator=g, device=DEV).to(I32), torch.zeros(1, dtype=I32, device=DEV)
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2))
    ang = torch.rand(512, d // 2, generator=g, device=DEV) * 6.28
    cos, sin = ang.cos(), ang.sin()
    lens, new = (torch.zeros(B, dtype=I32, device=DEV) for _ in range(2))
    qkv = torch.zeros(T, H, d, device=DEV, dtype=torch.bfloat16)
    logits, tokens = torch.zeros(T, V, device=DEV), torch.full((T,), -1, dtype=I32, device=DEV)
    plan, r = ch.plan_buffers(B, T, DEV), ch.logprob_buffers(T, 3, DEV)
    Q = torch.zeros(T, Hq, d, device=DEV, dtype=torch.bfloat16)
    out = torch.empty_like(Q), torch.empty(T, Hq, device=DEV)

    def step(stream=None):
        ch.plan(lens, new, free, begin, table, T, out=plan, stream=stream)
        ch.append8(qkv, wq, wk, cos, sin, plan.positions, plan.slots, K8, V8, sk, sv, EPS, out=Q, stream=stream)
        ch.attention8(Q, K8, V8, sk, sv, table, plan.cu_new, plan.kv_lens, out=out, stream=stream)
        ch.logprobs(logits, tokens, 3, out=r, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(side)          # no request has a token: nothing changes
    side.synchronize()
    assert bool(sk.isnan().all()) and int(plan.free_end) == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    keys, values = ([np.zeros((0, Hkv, d)) for _ in range(B)] for _ in range(2))
    grown = {"K": np.zeros((P, Hkv)), "V": np.zeros((P, Hkv))}
    for n, size in steps:
        new.copy_(torch.tensor(n, dtype=I32))
        qkv.copy_(torch.randn(T, H, d, generator=g, device=DEV) * size)
        logits.normal_(0, 3, generator=g)
        tokens.fill_(-1)
        tokens[:sum(n)] = torch.randint(0, V, (sum(n),), generator=g, device=DEV, dtype=I32)
        out[0].fill_(7.0)
        before = f(sk), f(sv)
        graph.replay()
        torch.cuda.synchronize()
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
        c, cu = sum(n), plan.cu_new.tolist()
        for name, old, now in (("K", before[0], f(sk)), ("V", before[1], f(sv))):
            grown[name] += np.where(np.isnan(old), 0, now > old)
        assert cu[-1] == c and bool((out[0][c:] == 7).all())
        if c == 0:
            lens.copy_(plan.kv_lens)
            continue
        pos = plan.positions[:c].cpu().numpy()
        q, k, v = S.qk_norm_rope(f(qkv[:c]), f(wq), f(wk), f(cos), f(sin), pos, Hq, EPS, False)
        assert (np.abs(f(Q[:c]) - q) <= 2.0 ** -8 * np.abs(q) + 2.0 ** -18 * np.abs(q).max(-1, keepdims=True)).all()
        for b in range(B):
            keys[b] = np.concatenate([keys[b], k[cu[b]:cu[b + 1]]])
            values[b] = np.concatenate([values[b], v[cu[b]:cu[b + 1]]])
        for name, cache, scale, want in (("K", K8, sk, keys), ("V", V8, sv, values)):
            for b in range(B):
                L = int(plan.kv_lens[b])
                assert L == len(want[b])
                at = np.arange(L)
                page = table[b].cpu().numpy()[at // 64]
                s = f(scale)[page]
                got = f(cache)[page, :, at % 64] * s[..., None]
                x, times = np.abs(want[b]), 1 + grown[name][page][..., None]
                tol = times * (1 + 2.0 ** -4) ** (times - 1) * (2.0 ** -4 * x + 2.0 ** -10 * s[..., None])
                if name == "K":
                    tol = tol + 2.0 ** -18 * x.max(-1, keepdims=True, initial=0.0)
                assert (np.abs(got - want[b]) <= tol).all(), (name, b)
        _compare(out[0][:c], out[1][:c], (Q[:c].clone(), K8, V8, sk, sv, table, plan.cu_new, plan.kv_lens), 1 / math.sqrt(d))
        z = logits[:c].double().log_softmax(-1)
        assert (r.logprob[:c].double() - z.gather(1, tokens[:c, None].long())[:, 0]).abs().max() < 2.0 ** -15
        assert torch.equal(r.top_index[:c].long(), logits[:c].topk(3).indices) and bool((r.top_index[c:] == -1).all())
        lens.copy_(plan.kv_lens)
        begin.copy_(plan.free_end)
    assert max(x.max() for x in grown.values()) > 1 and int(lens.max()) > 64      # scales that grew, more than once
    ch.close()
