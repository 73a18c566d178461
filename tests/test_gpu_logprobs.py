"""GPU log probabilities, entropy, alternatives and their gradient against the fp64 oracle.

Tolerances.  A term exp(z - m) is off by at most |y| 2^-23 (y = (z - m) log2 e and its product are rounded) + 2^-22 (the
exponential unit), the terms' weighted |y| by at most log2 V <= 18; a thread adds up to V / 256 / 2 <= 300 of them in a
row: 18 2^-23 + 2^-22 + 300 2^-24 < 2.1e-5 of the sum.  lse and logprob are off by that and two roundings of values as
large as the logits; the entropy, a quotient of two such sums of size <= 18 ln 2, by 13 times twice that."""
import math

import numpy as np
import pytest
import torch

from oracle import logp_oracle as L
from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32
BF, F32 = torch.bfloat16, torch.float32


def _layer():
    return sas.SasLayer(1, 1, 64, 64, 0)


def _chunk(T):
    return sas.SasChunk(1, 1, 1, 64, 1, 1, T)


def _logits(T, V, dtype, seed, std=3.0, pad=0, shift=0):
    """[T, V] of normal values inside a wider buffer whose other places hold NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    flat = torch.full((T * (V + pad) + shift,), math.nan, device=DEV, dtype=dtype)
    z = flat[shift:].view(T, V + pad)[:, :V]
    z.copy_(torch.randn(T, V, generator=g, device=DEV) * std)
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=I32)
    return z, tokens


def _check_rows(z, tokens, r, rows=None):
    zs = z.double().cpu().numpy()
    for t in range(z.shape[0]) if rows is None else rows:
        x = int(tokens[t])
        if x < 0:
            assert (float(r.logprob[t]), float(r.entropy[t]), float(r.lse[t])) == (0.0, 0.0, 0.0)
            continue
        lp, h, lse = L.row(zs[t], x)
        top = np.abs(zs[t][np.isfinite(zs[t])]).max() if np.isfinite(zs[t]).any() else 0.0
        tol = 2.1e-5 + 2 ** -22 * top
        got = float(r.lse[t])
        assert got == lse if math.isinf(lse) else abs(got - lse) <= tol, (t, got, lse)
        for a, b, c in ((float(r.logprob[t]), lp, tol), (float(r.entropy[t]), h, 26 * 2.1e-5)):
            assert (math.isnan(a) and math.isnan(b)) or a == b or abs(a - b) <= c, (t, a, b)


def _check_top(z, r, k, rows=None):
    zs = z.double().cpu().numpy()
    for t in range(z.shape[0]) if rows is None else rows:
        want = L.alternatives(zs[t], k)
        assert r.top_index[t].tolist() == want.tolist(), t
        lse = float(r.lse[t])
        for i, v in enumerate(want):
            got = float(r.top_logprob[t, i])
            ref = zs[t][v] - lse if v >= 0 else math.nan
            assert (math.isnan(got) and math.isnan(ref)) or got == ref or abs(got - ref) <= 1e-5 + 2 ** -22 * abs(zs[t][v]), (t, i)


# rows and columns: one, fewer than 16 bytes, a warp's rows, a block's, rows in parts; whether rows are 16-byte aligned
SIZES = [(1, 1, 0, 0), (1, 5, 0, 1), (9, 7, 0, 0), (3, 33, 5, 3), (40, 500, 0, 0), (17, 4096, 8, 0), (2, 4097, 0, 0), (33, 5003, 1, 1),
         (700, 4500, 0, 0), (5, 32003, 0, 0), (2, 151936, 0, 0), (1, 151935, 2, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,pad,shift", SIZES)
def test_rows(T, V, pad, shift, dtype):
    z, tokens = _logits(T, V, dtype, T + V, pad=pad, shift=shift)
    if T > 2:
        tokens[1] = -1
    layer, k = _layer(), min(V, 6)
    r = layer.token_logprobs(z, tokens)
    assert r.top_index is None
    rows = range(min(T, 40))
    _check_rows(z, tokens, r, rows)
    ch = _chunk(T)
    s = ch.logprobs(z, tokens, k)
    assert all(torch.equal(a, b) for a, b in zip(r[:3], s[:3]))
    _check_top(z, s, k, [t for t in rows if int(tokens[t]) >= 0])
    if T > 2:
        assert s.top_index[1].tolist() == [-1] * k and s.top_logprob[1].tolist() == [0.0] * k
    assert sas.sas_get_device_status(layer.h) == sas.sas_chunk_get_device_status(ch.h) == 0
    again = ch.logprobs(z, tokens, k, out=s)      # the same bits, and the workspace left as it was found
    assert again is s and all(torch.equal(a, b) for a, b in zip(again, ch.logprobs(z, tokens, k)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("per_sm,V", [(16, 4095), (16, 4097), (32, 4500), (32, 20011), (32, 32769)])
def test_many_rows(per_sm, V, dtype):
    # so many that a warp takes each, up to a length; hard rows among them
    T = per_sm * torch.cuda.get_device_properties(0).multi_processor_count + 3
    z, tokens = _logits(T, V, dtype, T + V, pad=3)
    z[0], z[2], z[3] = 0.25, -math.inf, torch.arange(V, device=DEV) % 5
    z[2, V - 1] = 1.0
    z[4, 7:V - 4] = math.nan
    z[5, : V - 3] = -math.inf
    tokens[1] = -1
    s = _chunk(T).logprobs(z, tokens, 32)
    r = _layer().token_logprobs(z, tokens)
    assert all(torch.equal(a, b) or torch.equal(a.isnan(), b.isnan()) and torch.equal(a[~a.isnan()], b[~b.isnan()]) for a, b in zip(r[:3], s[:3]))
    rows = [0, 2, 3, 5, 6, 7, 8, T // 2, T - 2, T - 1]
    _check_rows(z, tokens, r, rows)
    _check_top(z, s, 32, rows)
    few = _chunk(6).logprobs(z[:6], tokens[:6], 32)
    assert torch.equal(few.top_index, s.top_index[:6])


@pytest.mark.parametrize("V", [40, 500, 4500, 40000])
@pytest.mark.parametrize("k", [1, 2, 31, 32])
def test_alternatives_of_hard_rows(V, k):
    i = torch.arange(V, device=DEV, dtype=F32)
    rows = [i, -i, torch.zeros(V, device=DEV), (i % 7), (i * 37 % 11) - 5, torch.where(i % 2 == 0, 0.0, -0.0),
            torch.where(i < V - 3, -math.inf, i), torch.where(i == V // 2, 3e38, -3e38), -(i // 600), (i // 600)]
    z = torch.stack(rows).contiguous()
    tokens = torch.full((len(rows),), V // 2, device=DEV, dtype=I32)
    ch = _chunk(len(rows))
    for dtype in (F32, BF):
        r = ch.logprobs(z.to(dtype), tokens, k)
        _check_top(z.to(dtype), r, k, [t for t in range(len(rows)) if t != 7])
        assert r.top_index[7].tolist() == L.alternatives(z[7].cpu().numpy(), k).tolist()
        _check_rows(z.to(dtype), tokens, r, [1, 2, 3, 4, 5, 6, 8, 9])


@pytest.mark.parametrize("V", [33, 5000, 60000])
def test_infinities_and_nan(V):
    z, tokens = _logits(7, V, F32, 3)
    tokens[:] = 2
    z[0, 5] = math.nan
    z[1, 5] = math.inf
    z[2, :] = -math.inf
    z[3, 7:] = -math.inf                    # masked columns, and one column alone
    z[4, :] = -math.inf
    z[4, 2] = 1.5
    z[5, 2] = -math.inf                     # the token itself is masked
    z[6, :20] = math.nan
    ch, layer = _chunk(7), _layer()
    r = ch.logprobs(z, tokens, 5)
    for t in (0, 1, 6):
        assert all(math.isnan(float(x[t])) for x in r[:3])
    _check_rows(z, tokens, r, [2, 3, 4, 5])
    assert float(r.logprob[4]) == 0.0 and float(r.entropy[4]) == 0.0 and float(r.logprob[5]) == -math.inf
    for t in range(7):
        assert r.top_index[t].tolist() == L.alternatives(z[t].cpu().numpy(), 5).tolist()
    assert math.isnan(float(r.top_logprob[2, 0])) and r.top_logprob[4].tolist() == [0.0] + [-math.inf] * 4
    d = layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, torch.ones(7, device=DEV), torch.ones(7, device=DEV))
    assert torch.isfinite(d[[3, 4]]).all() and (d[3, 7:] == 0).all() and (d[4] == 0).all()
    assert torch.isnan(d[0]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,pad,shift", SIZES)
def test_gradient(T, V, pad, shift, dtype):
    """exp is off by |z - lse| 2^-23 + 2^-24 max(|z|, |lse|) + 2^-22 < 3e-5 for |z| < 45, and the factor beside it by a
    few roundings of its terms; then one rounding to the logits' type."""
    z, tokens = _logits(T, V, dtype, T + V + 1, pad=pad, shift=shift)
    if T > 2:
        tokens[1] = -1
    g = torch.Generator(device=DEV).manual_seed(5)
    gl, gh = torch.randn(T, generator=g, device=DEV), torch.randn(T, generator=g, device=DEV)
    layer = _layer()
    r = layer.token_logprobs(z, tokens)
    d = layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, gl, gh)
    assert d.dtype == dtype and d.shape == z.shape
    half = torch.finfo(dtype).eps / 2
    for t in range(min(T, 12)):
        x = int(tokens[t])
        if x < 0:
            assert (d[t] == 0).all()
            continue
        zt = z[t].double().cpu().numpy()
        args = zt, x, float(r.lse[t]), float(r.entropy[t]), float(gl[t]), float(gh[t])
        want, got = L.row_grad(*args), d[t].double().cpu().numpy()
        y = np.abs(zt - args[2])
        size = np.exp(zt - args[2]) * (abs(args[4]) + abs(args[5]) * (y + abs(args[3])))
        size[x] += abs(args[4]) * 2 ** -8
        assert (np.abs(got - want) <= 4e-5 * size + half * np.abs(want) + 1e-38).all()
    only = layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, gl)
    assert torch.equal(only, layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, gl, torch.zeros(T, device=DEV)))
    # outputs of other alignments, and the logits' own memory
    wide = torch.full((T, V + 3), 7.0, device=DEV, dtype=dtype)
    layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, gl, gh, out=wide[:, 1:V + 1])
    assert torch.equal(wide[:, 1:V + 1], d) and (wide[:, 0] == 7).all() and (wide[:, V + 1:] == 7).all()
    layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, gl, gh, out=z)
    assert torch.equal(z, d)
    assert sas.sas_get_device_status(layer.h) == 0


def test_gradient_against_differences_of_the_kernel():
    """Central differences of the fp32 kernel's own results, step 2^-4: the third derivative's h^2 / 6 < 7e-4, and
    2 (2.1e-5 + 26 2.1e-5) / 2^-3 < 1e-2 from the results' own errors."""
    z, tokens = _logits(3, 11, F32, 8, std=1.0)
    layer = _layer()
    gl, gh = torch.tensor([1.0, -0.5, 0.0], device=DEV), torch.tensor([0.5, 0.0, 1.0], device=DEV)
    r = layer.token_logprobs(z, tokens)
    d = layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, gl, gh)
    for v in range(11):
        e = torch.zeros(11, device=DEV)
        e[v] = 2.0 ** -4
        a, b = layer.token_logprobs((z + e).contiguous(), tokens), layer.token_logprobs((z - e).contiguous(), tokens)
        diff = (gl * (a.logprob - b.logprob) + gh * (a.entropy - b.entropy)) / 2 ** -3
        assert (diff - d[:, v]).abs().max() <= 1.1e-2


def test_tokens_outside_the_columns():
    z, tokens = _logits(4, 100, BF, 0)
    tokens[1], tokens[2] = 100, -2
    layer, ch = _layer(), _chunk(4)
    r = layer.token_logprobs(z, tokens)
    assert sas.sas_get_device_status(layer.h) == sas.SAS_ERR_INVALID_ARG
    assert r.logprob[1:3].tolist() == r.lse[1:3].tolist() == [0.0, 0.0]
    _check_rows(z, tokens, r, [0, 3])
    d = layer.token_logprobs_bwd(z, tokens, r.lse, r.entropy, torch.ones(4, device=DEV))
    assert sas.sas_get_device_status(layer.h) == sas.SAS_ERR_INVALID_ARG
    assert (d[1:3] == 0).all() and (d[0] != 0).any()
    s = ch.logprobs(z, tokens, 3)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG and s.top_index[1].tolist() == [-1] * 3


def test_captured_and_on_another_stream():
    z, tokens = _logits(6, 40000, BF, 2)
    ch, layer = _chunk(6), _layer()
    out = ch.logprob_buffers(6, 4, DEV)
    d = torch.empty_like(z)
    gl = torch.ones(6, device=DEV)
    ch.logprobs(z, tokens, 4)
    layer.token_logprobs_bwd(z, tokens, out.lse, out.entropy, gl)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ch.logprobs(z, tokens, 4, out=out)
        layer.token_logprobs_bwd(z, tokens, out.lse, out.entropy, gl, out=d)
    for seed in (3, 4):
        z2, t2 = _logits(6, 40000, BF, seed)
        z.copy_(z2)
        tokens.copy_(t2)
        g.replay()
        torch.cuda.synchronize()
        _check_rows(z2, t2, out)
        _check_top(z2, out, 4)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        r = ch.logprobs(z2, t2, 4, stream=side)
        e = layer.token_logprobs_bwd(z2, t2, r.lse, r.entropy, gl, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(r, out)) and torch.equal(e, d)


def test_refusals():
    z, tokens = _logits(4, 64, BF, 0)
    layer, ch = _layer(), _chunk(4)
    f = torch.ones(4, device=DEV)
    for bad in (z.half(), z[0], z.t(), z[:, ::2], z.cpu()):
        with pytest.raises(ValueError):
            ch.logprobs(bad, tokens, 1)
        with pytest.raises(ValueError):
            layer.token_logprobs(bad, tokens)
    for bad in (tokens.long(), tokens[:3], tokens.cpu(), tokens.repeat_interleave(2)[::2]):
        with pytest.raises(ValueError):
            ch.logprobs(z, bad, 1)
        with pytest.raises(ValueError):
            layer.token_logprobs_bwd(z, bad, f, f, f)
    for k in (33, 65):
        with pytest.raises(sas.SasError):
            ch.logprobs(z, tokens, k)
    with pytest.raises(sas.SasError):
        ch.logprobs(z[:, :3], tokens, 4)
    with pytest.raises(ValueError):
        ch.logprobs(z, tokens, 2, out=ch.logprob_buffers(4, 3, DEV))
    with pytest.raises(ValueError):
        ch.logprobs(z, tokens, 2, out=ch.logprob_buffers(3, 2, DEV))
    with pytest.raises(sas.SasError):
        ch.logprobs(torch.cat([z, z]), torch.cat([tokens, tokens]), 0)      # more than max_tokens
    with pytest.raises(ValueError):
        layer.token_logprobs_bwd(z, tokens, f[:3], f, f)
    with pytest.raises(ValueError):
        layer.token_logprobs_bwd(z, tokens, f, f, f, out=torch.empty(4, 64, device=DEV))
    with pytest.raises(sas.SasError):       # the logits' memory with other rows
        layer.token_logprobs_bwd(z.view(8, 32)[:4], tokens, f, f, f, out=z[:, :32])
    assert ch.logprobs(z, tokens, 32).top_index.shape == (4, 32)
