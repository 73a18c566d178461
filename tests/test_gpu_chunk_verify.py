"""GPU verification of drafted tokens against the oracle: accepted counts and tokens equal.

The inputs keep every comparison and quotient clear of fp32 rounding, or are meant to
tie exactly; `_clear` checks that before a test compares."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas
from tests import parity as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


def _case(counts, V, seed, near=0.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    B, n = len(counts), sum(counts)
    cu = torch.tensor([0] + np.cumsum(counts).tolist(), dtype=I32, device=DEV)
    z = torch.randn(n + B, V, generator=g, device=DEV) * 2
    keep = torch.ones(n + B, dtype=torch.bool, device=DEV)
    keep[cu[1:].long() + torch.arange(B, device=DEV)] = False
    target = torch.softmax(z, -1)
    draft = torch.softmax(z[keep] + near * torch.randn(n, V, generator=g, device=DEV), -1)
    tokens = torch.multinomial(draft, 1, generator=g)[:, 0].to(I32) if n else torch.zeros(0, dtype=I32, device=DEV)
    u = torch.rand(n, generator=g, device=DEV)
    noise = torch.empty(B, V, device=DEV).exponential_(1, generator=g) + 1e-6
    return tokens, cu, target, draft, u, noise


def _clear(case):
    """u q and p differ by more than one rounding wherever they are compared."""
    tokens, cu, target, draft, u, noise = case
    B = cu.shape[0] - 1
    keep = torch.ones(target.shape[0], dtype=torch.bool, device=DEV)
    keep[cu[1:].long() + torch.arange(B, device=DEV)] = False
    t = tokens.long()[:, None]
    p, q = target[keep].double().gather(1, t)[:, 0], draft.double().gather(1, t)[:, 0] * u.double()
    assert bool(((p - q).abs() > 2.0 ** -23 * p).all())


def _check(case, W, draft=True):
    tokens, cu, target, dr, u, noise = case
    ch = sas.SasChunk(cu.shape[0] - 1, 1, 1, 64, 1, 1, 1)
    a, out = ch.verify(tokens, cu, target, dr if draft else None, u, noise, W)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    a2, out2 = ch.verify(tokens, cu, target, dr if draft else None, u, noise, W)
    assert torch.equal(a, a2) and torch.equal(out, out2)
    ch.close()
    ra, rout = S.verify(tokens.cpu().numpy(), cu.tolist(), P.f64(target), P.f64(dr) if draft else None, P.f64(u), P.f64(noise), W)
    assert np.array_equal(a.cpu().numpy(), ra) and np.array_equal(out.cpu().numpy(), rout)
    return ra


@pytest.mark.parametrize("V", [1, 2, 3, 31, 1000, 1023, 2048, 4099, 32003])
def test_vocabularies(V):
    case = _case([3, 0, 5, 1, 2], V, seed=V)
    if V > 1:
        _clear(case)
    _check(case, 5)


@pytest.mark.parametrize("counts,W", [([0], 0), ([0, 0, 0], 4), ([70], 70), ([33, 1, 64, 0, 31], 64), ([1] * 300, 1), ([2, 3] * 40, 9)])
def test_draft_counts(counts, W):
    case = _case(counts, 257, seed=len(counts), near=0.2)
    _clear(case)
    _check(case, W)


def test_all_accepted_none_accepted_and_certain_drafts():
    tokens, cu, target, draft, u, noise = _case([4] * 6, 500, seed=1)
    assert _check((tokens, cu, target, draft, torch.zeros_like(u), noise), 4).tolist() == [4] * 6
    none = target.clone()
    keep = torch.ones(30, dtype=torch.bool, device=DEV)
    keep[cu[1:].long() + torch.arange(6, device=DEV)] = False
    rows = keep.nonzero()[:, 0]
    none[rows, tokens.long()] = 0
    assert _check((tokens, cu, none, draft, u, noise), 4).tolist() == [0] * 6
    for s in range(3):
        _check(_case([6] * 20, 8, seed=s, near=0.01), 6, draft=False)


def test_rows_of_any_stride_and_alignment():
    tokens, cu, target, draft, u, noise = _case([3, 2], 1000, seed=2)
    want = None
    for pad, off in ((0, 0), (24, 0), (24, 4), (3, 0), (3, 1)):
        def place(t):
            wide = torch.full((t.shape[0], 1000 + pad + off), float("nan"), device=DEV)
            wide[:, off:off + 1000] = t
            return wide[:, off:off + 1000]
        ch = sas.SasChunk(2, 1, 1, 64, 1, 1, 1)
        got = ch.verify(tokens, cu, place(target), place(draft), u, place(noise), 3)
        ch.close()
        want = want or got
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    _check((tokens, cu, target, draft, u, noise), 3)


def test_a_large_row_takes_the_last_and_first_columns():
    # one certain winner at each end of a row that many blocks share, and equal ones: the lowest
    V = 151936
    for hot in ([0], [V - 1], [77777], [5, 6, V - 1], [2047, 2048], [100000, 140000]):
        p = torch.full((1, V), 1e-9, device=DEV)
        p[0, hot] = 0.1
        case = (torch.zeros(0, dtype=I32, device=DEV), torch.tensor([0, 0], dtype=I32, device=DEV), p,
                torch.zeros(0, V, device=DEV), torch.zeros(0, device=DEV), torch.ones(1, V, device=DEV))
        ch = sas.SasChunk(1, 1, 1, 64, 1, 1, 1)
        a, out = ch.verify(*case, 0)
        ch.close()
        assert a.tolist() == [0] and out.tolist() == [[hot[0]]]


def test_empty_residual_falls_back_to_the_target():
    V = 5000
    tokens, cu, target, draft, u, noise = _case([2, 2], V, seed=4)
    rows = torch.tensor([0, 1, 3, 4], device=DEV)
    draft = target[rows].clone()
    draft[0] = torch.nextafter(draft[0], torch.ones_like(draft[0]))   # p < q everywhere, then p = q
    target[0, int(tokens[0])] = 0                                      # rejected at once
    target[3, int(tokens[2])] = 0
    draft[2, int(tokens[2])] = 1.0
    u[0] = u[2] = 0.5
    _check((tokens, cu, target, draft, u, noise), 2)


def test_non_finite_zero_and_denormal_values():
    # NaN and zero weights and non-positive noise are never chosen; tiny ones compare rightly
    V = 4096
    target = torch.full((4, V), float("nan"), device=DEV)
    noise = torch.ones(4, V, device=DEV)
    target[0, 100], target[0, 200] = 1e-42, 2e-42
    target[1, 9], target[1, 10], noise[1, 9] = 0.5, 0.25, 0.0
    target[2, 9], target[2, 3000], noise[2, 9], noise[2, 3000] = 0.5, 0.5, -1.0, 1e-38
    target[3, 7], target[3, 8], noise[3] = 1e-30, 3e-30, 1e-12
    ch = sas.SasChunk(4, 1, 1, 64, 1, 1, 1)
    empty = torch.zeros(0, dtype=I32, device=DEV)
    a, out = ch.verify(empty, torch.zeros(5, dtype=I32, device=DEV), target, None, empty.float(), noise, 0)
    assert out[:, 0].tolist() == [200, 10, 3000, 8] and sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    target[1] = 0
    a, out = ch.verify(empty, torch.zeros(5, dtype=I32, device=DEV), target, None, empty.float(), noise, 0)
    assert out[:, 0].tolist() == [200, -1, 3000, 8]
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
    ch.close()


def test_tokens_are_distributed_as_the_target():
    B, V = 200000, 5
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    p = torch.tensor([.05, .1, .2, .25, .4], device=DEV)
    q = torch.tensor([.4, .25, .2, .1, .05], device=DEV)
    tokens = torch.multinomial(q, B, True, generator=g).to(I32)
    total = torch.zeros(V, dtype=torch.int64, device=DEV)
    ch = sas.SasChunk(8000, 1, 1, 64, 1, 1, 1)
    for k in range(0, B, 8000):
        _, out = ch.verify(tokens[k:k + 8000], torch.arange(8001, dtype=I32, device=DEV), p.repeat(16000, 1), q.repeat(8000, 1),
                           torch.rand(8000, generator=g, device=DEV), torch.empty(8000, V, device=DEV).exponential_(1, generator=g), 1)
        total += torch.bincount(out[:, 0].long(), minlength=V)
    ch.close()
    f, p = P.f64(total) / B, P.f64(p)
    assert np.all(np.abs(f - p) < 5 * np.sqrt(p * (1 - p) / B))   # five standard deviations


def test_bad_offsets_and_tokens():
    tokens, cu, target, draft, u, noise = _case([2, 2, 2], 50, seed=6)
    u.zero_()   # everything valid is accepted
    ch = sas.SasChunk(3, 1, 1, 64, 1, 1, 1)
    t = tokens.clone()
    t[1], t[2] = 50, -1
    a, out = ch.verify(t, cu, target, draft, u, noise, 2)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
    assert a.tolist() == [1, 0, 2] and bool((out[0, :2] >= 0).all()) and out[0, 2] == -1 and out[1, 1:].tolist() == [-1, -1]
    for bad in ([0, 4, 3, 6], [0, 2, 7, 7], [-1, 2, 4, 6]):
        a, out = ch.verify(tokens, torch.tensor(bad, dtype=I32, device=DEV), target, draft, u, noise, 2)
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
        for b in range(3):
            ok = 0 <= bad[b] <= bad[b + 1] <= 6 and bad[b + 1] - bad[b] <= 2
            assert ok or (a[b] == 0 and out[b].tolist() == [-1] * 3)
    a, out = ch.verify(tokens, cu, target, draft, u, noise, 2)   # the workspace is as before
    assert a.tolist() == [2, 2, 2] and sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()


def test_refusals():
    tokens, cu, target, draft, u, noise = _case([2, 1], 50, seed=6)
    ch = sas.SasChunk(1, 1, 1, 64, 1, 1, 1)
    with pytest.raises(sas.SasError, match="num_seqs"):
        ch.verify(tokens, cu, target, draft, u, noise, 2)
    ch.close()
    ch = sas.SasChunk(2, 1, 1, 64, 1, 1, 1)
    with pytest.raises(ValueError, match="target"):
        ch.verify(tokens, cu, target[1:], draft, u, noise, 2)
    with pytest.raises(ValueError, match="draft"):
        ch.verify(tokens, cu, target, draft.half(), u, noise, 2)
    with pytest.raises(ValueError, match="columns"):
        ch.verify(tokens, cu, target, draft, u, noise.t().contiguous().t(), 2)
    with pytest.raises(sas.SasError, match="stride"):
        ch.verify(tokens, cu, target[:1].expand(5, 50), draft, u, noise, 2)
    assert sas.sas_chunk_launch_count(ch.h) == 0
    ch.close()
