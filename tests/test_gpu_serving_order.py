"""Kernels that come in before the one ahead has ended see what it wrote, and write after it has read.

Two sets of inputs take turns in the same buffers, written by other kernels right before
each call and read by others right after it; the results are those of the same calls with
the device waited for in between."""
import pytest
import torch

from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32, BF = torch.int32, torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ints(x, dtype=I32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(BF)


def _turns(write, call, sets, waits):
    """write(buffers, set) and call() in turn; the outputs of every call, cloned by kernels behind it."""
    slow = torch.randn(2048, 2048, device=DEV)
    got = []
    for i in range(10):
        torch.mm(slow, slow)          # the device has work: the calls below are queued, not waited for
        write(sets[i % 2])
        if waits:
            torch.cuda.synchronize()
        out = call()
        if waits:
            torch.cuda.synchronize()
        got.append([t.clone() for t in out])
    torch.cuda.synchronize()
    return got


def _check(buffers, sets, call):
    def write(values):
        for b, v in zip(buffers, values):
            b.copy_(v)
    free, waited = _turns(write, call, sets, False), _turns(write, call, sets, True)
    for a, b in zip(free, waited):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert any(not torch.equal(x, y) for x, y in zip(free[0], free[1]))   # the sets do differ


def _tables(n, rot):
    ang = torch.arange(n, device=DEV)[:, None] / 100.0 ** (torch.arange(0, rot, 2, device=DEV) / rot)
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


@pytest.mark.parametrize("d", [64, 128])
def test_norm_rope_and_its_gradient(d):
    B, N, H, Hkv = 1, 1500, 4, 2
    layer = sas.SasLayer(B, H, N, d, 1, Hkv=Hkv)
    sets = []
    for s in range(2):
        g = _gen(s)
        pos = torch.randint(0, 64, (B, N), generator=g, device=DEV, dtype=I32)
        sets.append([_normal(g, B, N, H + 2 * Hkv, d), _normal(g, d), _normal(g, d), *[t * (1 + s) for t in _tables(64, d)], pos,
                     _normal(g, B, H, N, d), _normal(g, B, Hkv, N, d), _normal(g, B, Hkv, N, d)])
    x = [t.clone() for t in sets[0]]
    _check(x, sets, lambda: [*layer.qk_norm_rope(*x[:5], positions=x[5]), *layer.qk_norm_rope_bwd(*x[:5], *x[6:], positions=x[5])])
    layer.close()


@pytest.mark.parametrize("d", [64, 128])
def test_plan_append_attention(d):
    Hq, Hkv, B, T, P = 4, 2, 5, 400, 120
    ch = sas.SasChunk(B, Hq, Hkv, d, 32, P, T)
    sets = []
    for s, (seq, new) in enumerate([([100, 0, 700, 63, 64], [1, 130, 5, 66, 0]), ([9, 640, 64, 0, 250], [200, 3, 64, 1, 17])]):
        g = _gen(s)
        table = torch.full((B, 32), -1, dtype=I32, device=DEV)
        perm = torch.randperm(P, generator=g, device=DEV).to(I32)
        at = 0
        for b, n in enumerate(seq):
            k = -(-n // 64)
            table[b, :k] = perm[at:at + k]
            at += k
        sets.append([_ints(seq), _ints(new), perm.roll(-at), _ints([0]), table, _normal(g, T, Hq + 2 * Hkv, d), _normal(g, d),
                     _normal(g, d), *_tables(1000, d), _normal(g, P, Hkv, 64, d), _normal(g, P, Hkv, 64, d)])
    x = [t.clone() for t in sets[0]]
    plan = ch.plan_buffers(B, T, torch.device(DEV))
    q = torch.zeros(T, Hq, d, device=DEV, dtype=BF)
    o, lse = torch.zeros_like(q), torch.zeros(T, Hq, device=DEV)

    def call():
        o.zero_()
        lse.zero_()
        q.zero_()
        p = ch.plan(*x[:4], x[4], T, out=plan)
        ch.append(*x[5:10], p.positions, p.slots, x[10], x[11], out=q)
        ch.attention(q, x[10], x[11], x[4], p.cu_new, p.kv_lens, out=(o, lse))
        return [*plan, x[4], q, x[10], x[11], o, lse]

    _check(x, sets, call)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()


def test_verify():
    B, W, V = 6, 4, 20000
    ch = sas.SasChunk(B, 1, 1, 64, 1, 1, 1)
    sets = []
    for s, counts in enumerate([[4, 0, 2, 4, 1, 4], [1, 4, 4, 3, 3, 0]]):
        g = _gen(s)
        n = sum(counts)
        rows = lambda k: torch.softmax(torch.randn(k, V, generator=g, device=DEV), -1)  # noqa: E731
        cu = [0]
        for c in counts:
            cu.append(cu[-1] + c)
        sets.append([torch.randint(0, V, (n,), generator=g, device=DEV, dtype=I32), _ints(cu), rows(n + B), rows(n),
                     torch.rand(n, generator=g, device=DEV) * 0.5, -torch.rand(B, V, generator=g, device=DEV).log()])
    x = [t.clone() for t in sets[0]]
    _check(x, sets, lambda: list(ch.verify(*x, W)))
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()
