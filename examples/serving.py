"""One attention layer served and trained through the package's entry points.

    python examples/serving.py            # prompts in chunks, SAS decode, a drafted step; times of each
    python examples/serving.py --train    # norm + rotation, SAS attention, and back to the projection

Serving keeps one paged cache for all requests:
  * prompts enter in chunks, together with whatever else runs: SasChunk.plan gives pages
    and slots, append norms, rotates and writes the cache, attention runs the new tokens;
  * SasDecoder.summarize and step continue on the same cache with SAS selection;
  * drafted tokens run as a chunk of several tokens per request; SasChunk.verify accepts a
    prefix, and the lengths go back to what was accepted.
Weights and inputs are random: the example shows the calls and their order.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_13141_gb300 import sas  # noqa: E402

I32, BF = torch.int32, torch.bfloat16


def rotation_tables(max_pos, rot, theta=1e6, device="cuda"):
    """cos and sin [max_pos, rot / 2], computed in fp64."""
    inv = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    ang = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] * inv
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


class Server:
    """One layer's cache, page table and handles."""

    def __init__(self, requests, Hq, Hkv, d, max_len, chunk, topk=32, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.g, self.dev, self.B, self.chunk = g, device, requests, chunk
        self.shape = (Hq, Hkv, d)
        blocks = -(-max_len // 64)
        pages = requests * blocks
        self.step = sas.SasChunk(requests, Hq, Hkv, d, blocks, pages, chunk)
        self.dec = sas.SasDecoder(requests, Hq, Hkv, d, topk, blocks, pages)
        self.K = torch.zeros(pages, Hkv, 64, d, device=device, dtype=BF)
        self.V = torch.zeros_like(self.K)
        self.table = torch.full((requests, blocks), -1, device=device, dtype=I32)
        self.lens = torch.zeros(requests, device=device, dtype=I32)
        self.held = torch.zeros_like(self.lens)   # tokens whose pages each request holds
        self.free = torch.randperm(pages, generator=g, device=device).to(I32)
        self.taken = torch.zeros(1, device=device, dtype=I32)
        self.cos, self.sin = rotation_tables(max_len, d, device=device)
        self.wq = (1 + 0.1 * torch.randn(d, generator=g, device=device)).to(BF)
        self.wk = (1 + 0.1 * torch.randn(d, generator=g, device=device)).to(BF)
        self.sel_q = (0.02 * torch.randn(Hkv, d, Hq // Hkv * d, generator=g, device=device)).to(BF)
        self.sel_k = (0.02 * torch.randn(Hkv, d, d, generator=g, device=device)).to(BF)
        self.Ksum = torch.zeros(requests, Hkv, blocks, d, device=device, dtype=BF)

    def projection(self, tokens):
        """Stands in for the layer's fused QKV projection."""
        Hq, Hkv, d = self.shape
        return torch.randn(tokens, Hq + 2 * Hkv, d, generator=self.g, device=self.dev).to(BF)

    def enter(self, qkv, new_lens):
        """The new tokens of every request (rows of qkv in request order, `new_lens` each; spare rows at the end) into
        the cache.  Returns the plan and the queries.

        A plan that does not fit (no pages left, a request past its table) is refused whole, and the status word of
        the handle says so: the lengths and pages stay, and self.entered, the tokens that the last plan let in, is zero.
        Rows of no token are zero."""
        p = self.step.plan(self.lens, new_lens, self.free, self.taken, self.table, qkv.shape[0], held_lens=self.held)
        Q = torch.zeros(qkv.shape[0], *self.shape[::2], device=self.dev, dtype=BF)
        self.step.append(qkv, self.wq, self.wk, self.cos, self.sin, p.positions, p.slots, self.K, self.V, out=Q)
        self.lens, self.taken, self.entered = p.kv_lens, p.free_end, p.cu_new[-1]
        self.held = torch.maximum(self.held, self.lens)
        return p, Q

    def forward(self, qkv, new_lens):
        """enter(), and the dense attention of the new tokens."""
        p, Q = self.enter(qkv, new_lens)
        O = torch.zeros_like(Q)
        self.step.attention(Q, self.K, self.V, self.table, p.cu_new, p.kv_lens, out=(O, None))
        return O

    def summarize(self):
        """The selector's summaries of the full blocks, which steps of several tokens leave to this call."""
        self.dec.summarize(self.K, self.table, self.lens, self.sel_k, self.Ksum)

    def prefill(self, prompts):
        """Prompts (a [tokens, heads, d] projection each) in steps of at most `chunk` tokens over all requests.
        Returns each prompt's attention output.  Raises RuntimeError when a step is refused (the host waits for each
        step's plan); the steps before it stand, and self.lens counts their tokens."""
        done, out = [0] * len(prompts), [[] for _ in prompts]
        while any(d < p.shape[0] for d, p in zip(done, prompts)):
            room, take = self.chunk, []
            for d, p in zip(done, prompts):
                take.append(min(room, p.shape[0] - d))
                room -= take[-1]
            qkv = torch.cat([p[d:d + n] for p, d, n in zip(prompts, done, take)])
            O = self.forward(qkv, torch.tensor(take, device=self.dev, dtype=I32))
            if int(self.entered) != sum(take):
                self.summarize()
                raise RuntimeError("no pages, or no room in a request's table, for a chunk of the prompts")
            at = 0
            for b, n in enumerate(take):
                out[b].append(O[at:at + n])
                at += n
                done[b] += n
        self.summarize()
        return [torch.cat(o) for o in out]

    def decode(self, qkv):
        """One token per request with SAS selection.  qkv [requests, heads, d].  A refused step gives zeros."""
        p, Q = self.enter(qkv, torch.ones_like(self.lens))
        O, _, kept = self.dec.step(Q, self.K, self.V, self.table, p.kv_lens, Wq=self.sel_q, Wk=self.sel_k, Ksum=self.Ksum)
        return torch.where(self.entered > 0, O, 0), kept

    def drafted(self, qkv, drafts, draft_probs, target_probs_of):
        """A step over `drafts` [requests, n] and the token before them: target_probs_of(O) gives the n + 1 target
        rows of every request.  Keeps the accepted tokens; returns (accepted, tokens): 0 and -1 throughout from a
        refused step, which keeps nothing.  The drafts are attended densely, also where decode() would select."""
        B, n = drafts.shape
        lens = self.lens
        O = self.forward(qkv, torch.full_like(lens, n + 1))
        cu = torch.arange(0, (B + 1) * n, n, device=self.dev, dtype=I32)
        target = target_probs_of(O)
        u = torch.rand(B * n, generator=self.g, device=self.dev)
        noise = torch.empty(B, target.shape[1], device=self.dev).exponential_(1, generator=self.g)
        accepted, tokens = self.step.verify(drafts.reshape(-1), cu, target, draft_probs, u, noise, n)
        granted = self.entered > 0
        accepted, tokens = torch.where(granted, accepted, 0), torch.where(granted, tokens, -1)
        # the cache keeps the token before the drafts and the accepted ones; pages opened for the rest stay
        # with the request, and their slots are written again by the next step
        self.lens = lens + (1 + accepted) * granted
        self.summarize()
        return accepted, tokens

    def close(self):
        self.step.close()
        self.dec.close()


def train_step(qkv, wq, wk, cos, sin, Hq, Hkv, topk, scores, dO, layer=None):
    """Projection -> norm + rotation -> SAS attention and back.  qkv [B, N, Hq + 2 Hkv, d]; returns (O, dqkv, dwq, dwk,
    dscores)."""
    B, N, _, d = qkv.shape
    own = layer is None
    if own:
        layer = sas.SasLayer(B, Hq, N, d, topk, Hkv=Hkv)
    Q, K, V = layer.qk_norm_rope(qkv, wq, wk, cos, sin)
    O, LSE, idx, logg = layer.attention(Q, K, V, scores)
    dQ, dK, dV, _, dscores = layer.attention_bwd(Q, K, V, O, LSE, dO, scores, idx, logg, want_ds=True)
    dqkv, dwq, dwk = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, dQ, dK, dV)
    if own:
        layer.close()
    return O, dqkv, dwq, dwk, dscores


def _timed(name, fn):
    torch.cuda.synchronize()
    t = time.perf_counter()
    r = fn()
    torch.cuda.synchronize()
    print(f"{name:44s} {(time.perf_counter() - t) * 1e3:9.3f} ms")
    return r


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--train", action="store_true")
    a = ap.parse_args()
    torch.manual_seed(0)
    if a.train:
        B, N, Hq, Hkv, d, topk = 1, 8192, 32, 8, 128, 32
        qkv = torch.randn(B, N, Hq + 2 * Hkv, d, device="cuda").to(BF)
        w = torch.ones(d, device="cuda", dtype=BF)
        cos, sin = rotation_tables(N, d)
        scores = torch.randn(B, Hkv, N, -(-N // 64), device="cuda")
        dO = torch.randn(B, Hq, N, d, device="cuda").to(BF)
        layer = sas.SasLayer(B, Hq, N, d, topk, Hkv=Hkv)
        for name in ("first step", "second step"):
            _timed(f"{name}, {N} tokens", lambda: train_step(qkv, w, w, cos, sin, Hq, Hkv, topk, scores, dO, layer))
        layer.close()
        return
    Hq, Hkv, d, V = 32, 8, 128, 32000
    prompts = [5000, 300, 12000, 64, 2111, 1, 8000, 700]
    s = Server(len(prompts), Hq, Hkv, d, 16384, 4096)
    x = [s.projection(n) for n in prompts]
    _timed(f"prefill of {sum(prompts)} tokens in chunks of {s.chunk}", lambda: s.prefill(x))
    for name in ("first", "second"):
        y = s.projection(len(prompts))
        _timed(f"{name} SAS decode step of {len(prompts)} requests", lambda: s.decode(y))
    n = 4
    draft_probs = torch.softmax(torch.randn(len(prompts) * n, V, device="cuda"), -1)
    drafts = torch.multinomial(draft_probs, 1).to(I32).view(len(prompts), n)
    head = torch.randn(Hq * d, V, device="cuda", dtype=BF) * 0.02
    probs = lambda O: torch.softmax((O.reshape(O.shape[0], -1) @ head).float(), -1)  # noqa: E731
    y = s.projection(len(prompts) * (n + 1))
    probs(torch.zeros(1, Hq, d, device="cuda", dtype=BF))   # the library's first call is not the step's
    accepted, tokens = _timed(f"step of {n} drafts per request, verified", lambda: s.drafted(y, drafts, draft_probs, probs))
    print("accepted", accepted.tolist(), "next tokens", tokens.gather(1, accepted.long()[:, None])[:, 0].tolist())
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_OK and sas.sas_decode_get_device_status(s.dec.h) == sas.SAS_OK
    s.close()


if __name__ == "__main__":
    main()
