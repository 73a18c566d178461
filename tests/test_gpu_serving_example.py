"""The example's paths, small: served requests and a training step against fp64 references of the whole path.

Bounds: the path's tensors are rounded to bf16 at most six times (q, k, P, O and, going back, dO's products and dqkv),
each 2^-8 of its values, and independent: in the 2-norm well under 2^-5 of the result, which a wrong mask, position,
page or missing term passes many times over."""
import math

import numpy as np
import pytest
import torch

from examples import serving as X
from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas
from tests import parity as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rel(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def _dense(s, x, upto=None):
    """fp64 norm + rotation and causal attention of a whole request; rows from `upto` on only."""
    Hq, Hkv, d = s.shape
    T = x.shape[0]
    q, k, v = S.qk_norm_rope(P.f64(x), P.f64(s.wq), P.f64(s.wk), P.f64(s.cos), P.f64(s.sin), np.arange(T), Hq, 1e-6, False)
    out = np.zeros((T, Hq, d))
    for t in range(upto or 0, T):
        for h in range(Hq):
            z = k[:t + 1, h // (Hq // Hkv)] @ q[t, h] / math.sqrt(d)
            e = np.exp(z - z.max())
            out[t, h] = e @ v[:t + 1, h // (Hq // Hkv)] / e.sum()
    return out


def test_prompts_decode_and_drafts_follow_one_cache():
    prompts = [150, 1, 64, 63, 97]
    s = X.Server(len(prompts), 4, 2, 64, 320, 70, topk=32)   # 32 blocks kept of at most 5: SAS decode is dense
    x = [s.projection(n) for n in prompts]
    out = s.prefill(x)
    for b in range(len(prompts)):
        assert _rel(P.f64(out[b]), _dense(s, x[b])) < 2.0 ** -5
    for _ in range(3):
        y = s.projection(len(prompts))
        O, kept = s.decode(y)
        x = [torch.cat((a, y[b:b + 1])) for b, a in enumerate(x)]
        for b in range(len(prompts)):
            assert _rel(P.f64(O[b]), _dense(s, x[b], x[b].shape[0] - 1)[-1]) < 2.0 ** -5
    # four drafts per request, twice: what is rejected leaves nothing behind, and its pages are used again
    V, n, B = 50, 4, len(prompts)
    for step in range(3):
        probs = torch.softmax(torch.randn(B * n, V, generator=s.g, device=DEV), -1)
        drafts = torch.multinomial(probs, 1, generator=s.g).to(torch.int32).view(B, n)
        y = s.projection(B * (n + 1))
        seen = []

        def target(O):
            seen.append(O)
            t = torch.softmax(torch.randn(B * (n + 1), V, generator=s.g, device=DEV), -1).view(B, n + 1, V)
            t[:, :n] = 0.5 * t[:, :n] + 0.5 * probs.view(B, n, V)
            return t.view(-1, V)

        before = s.lens.clone()
        accepted, tokens = s.drafted(y, drafts, probs, target)
        rows = [torch.cat((a, y[b * (n + 1):(b + 1) * (n + 1)])) for b, a in enumerate(x)]
        for b in range(B):
            want = _dense(s, rows[b], x[b].shape[0])[x[b].shape[0]:]
            assert _rel(P.f64(seen[0].view(B, n + 1, 4, 64)[b]), want) < 2.0 ** -5
            a = int(accepted[b])
            assert tokens[b, :a].tolist() == drafts[b, :a].tolist() and 0 <= int(tokens[b, a]) < V
            x[b] = rows[b][:x[b].shape[0] + 1 + a]
        assert torch.equal(s.lens, before + 1 + accepted)
        y = s.projection(B)
        O, _ = s.decode(y)
        x = [torch.cat((a, y[b:b + 1])) for b, a in enumerate(x)]
        for b in range(B):
            assert _rel(P.f64(O[b]), _dense(s, x[b], x[b].shape[0] - 1)[-1]) < 2.0 ** -5
    # no page is lost: taken pages are exactly the tables' entries
    held = s.table[s.table >= 0].tolist()
    assert len(held) == len(set(held)) == int(s.taken) == int(((s.held + 63) // 64).sum())
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_OK and sas.sas_decode_get_device_status(s.dec.h) == sas.SAS_OK
    s.close()


def test_training_step_gradients():
    # every block kept, hard gates: the attention is the dense causal one, whose whole chain autograd runs in fp64
    B, N, Hq, Hkv, d = 1, 200, 4, 2, 128
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    qkv = torch.randn(B, N, Hq + 2 * Hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2))
    cos, sin = X.rotation_tables(N, d, device=DEV)
    dO = torch.randn(B, Hq, N, d, generator=g, device=DEV).to(torch.bfloat16)
    scores = torch.randn(B, Hkv, N, -(-N // 64), generator=g, device=DEV)
    layer = sas.SasLayer(B, Hq, N, d, 8, Hkv=Hkv, mode=sas.SAS_MODE_INFER_HARD)
    O, dqkv, dwq, dwk, _ = X.train_step(qkv, wq, wk, cos, sin, Hq, Hkv, 8, scores, dO, layer)
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    layer.close()
    x, a, b = (t.double().requires_grad_() for t in (qkv, wq, wk))
    c, s = cos.double()[:, None], sin.double()[:, None]

    def turned(z, w):
        z = z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        lo, hi = z[..., :d // 2], z[..., d // 2:]
        return torch.cat((lo * c - hi * s, hi * c + lo * s), -1).transpose(1, 2)

    q, k, v = turned(x[:, :, :Hq], a), turned(x[:, :, Hq:Hq + Hkv], b), x[:, :, Hq + Hkv:].transpose(1, 2)
    k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
    z = (q @ k.transpose(2, 3) / math.sqrt(d)).masked_fill(torch.ones(N, N, device=DEV).triu(1).bool(), -math.inf)
    out = torch.softmax(z, -1) @ v
    out.backward(dO.double())
    assert _rel(P.f64(O), P.f64(out)) < 2.0 ** -5
    for got, want in ((dqkv, x.grad), (dwq, a.grad), (dwk, b.grad)):
        assert _rel(P.f64(got), P.f64(want)) < 2.0 ** -5
