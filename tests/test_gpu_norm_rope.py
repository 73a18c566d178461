"""GPU parity of the per-head norm + rotation (forward, gradient, into cache pages)
against the fp64 oracle.

Bounds.  Outputs are one bf16 rounding (2^-8 |y|) of fp32 arithmetic on the inputs:
a sum of d squares in a tree, a reciprocal square root (2 ulp), three products and a
pair sum, each 2^-24 of terms no larger than the row's largest, so 2^-17 of that.
The gradient adds a mean of d products, of terms up to r (|u| + |xh| mean|u xh|).
dw sums at most 2^7 terms a lane one after the other and then trees: 2^-17 of the
sum of the terms' sizes, their own roundings included."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas
from tests import parity as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(torch.bfloat16)


def _tables(max_pos, rot, theta=1e4):
    ang = torch.arange(max_pos, device=DEV, dtype=torch.float64)[:, None] * \
        theta ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def _weights(g, d):
    return _normal(g, d), _normal(g, d)


def _close(got, want, scale, what):
    err = np.abs(P.f64(got) - want)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * scale
    assert np.all(err <= tol), f"{what}: worst {np.max(err - tol):.3g} over the bound"


def _row_scale(qkv, w, Hq, eps=EPS):
    """Largest |z| of each row, [T, H, 1]."""
    H = qkv.shape[1]
    Hkv = (H - Hq) // 2
    r = 1 / np.sqrt((qkv ** 2).mean(-1, keepdims=True) + eps)
    ws = np.stack([w[0]] * Hq + [w[1]] * Hkv + [np.ones_like(w[0])] * Hkv)
    return np.abs(qkv * r * ws).max(-1, keepdims=True)


CASES = [
    # B, N, Hq, Hkv, d, rot, interleaved, pad of the token stride
    (1, 1, 1, 1, 64, 64, False, 0),
    (1, 1, 8, 1, 128, 128, True, 8),
    (2, 65, 4, 2, 128, 128, False, 0),
    (2, 37, 6, 3, 64, 16, False, 64),
    (1, 70, 5, 5, 128, 48, True, 0),
    (3, 19, 12, 12, 64, 32, True, 24),
    (1, 33, 32, 8, 128, 64, False, 0),
]


def _inputs(B, N, Hq, Hkv, d, rot, pad, seed=0):
    g = _gen(seed)
    H = Hq + 2 * Hkv
    wide = _normal(g, B, N, H * d + pad, std=2.0)
    qkv = wide[:, :, :H * d].unflatten(-1, (H, d))
    return g, qkv, *_weights(g, d), *_tables(N + 5, rot)


@pytest.mark.parametrize("B,N,Hq,Hkv,d,rot,inter,pad", CASES)
@pytest.mark.parametrize("given", [False, True])
def test_forward_and_gradient_match_the_oracle(B, N, Hq, Hkv, d, rot, inter, pad, given):
    g, qkv, wq, wk, cos, sin = _inputs(B, N, Hq, Hkv, d, rot, pad, seed=N)
    H = Hq + 2 * Hkv
    pos = torch.randint(0, N + 5, (B, N), generator=g, device=DEV, dtype=torch.int32) if given else None
    layer = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    Q, K, V = layer.qk_norm_rope(qkv, wq, wk, cos, sin, pos, EPS, inter)
    dQ, dK, dV = _normal(g, *Q.shape), _normal(g, *K.shape), _normal(g, *V.shape)
    dqkv, dwq, dwk = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, dQ, dK, dV, pos, EPS, inter)
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    again = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, dQ, dK, dV, pos, EPS, inter)
    assert all(torch.equal(a, b) for a, b in zip((dqkv, dwq, dwk), again))
    layer.close()

    p = (pos.cpu().numpy() if given else np.tile(np.arange(N), (B, 1))).reshape(-1)
    x = P.f64(qkv).reshape(B * N, H, d)
    w = (P.f64(wq), P.f64(wk))
    tabs = (P.f64(cos), P.f64(sin))
    want = S.qk_norm_rope(x, *w, *tabs, p, Hq, EPS, inter)
    zmax = _row_scale(x, w, Hq)
    bnhd = lambda t: P.f64(t.transpose(1, 2).reshape(B * N, -1, d))  # noqa: E731
    for got, ref, sc in zip((Q, K), want, (zmax[:, :Hq], zmax[:, Hq:Hq + Hkv])):
        _close(torch.from_numpy(bnhd(got)), ref, sc, "forward")
    assert np.array_equal(bnhd(V), want[2])

    dY = np.concatenate([bnhd(t) for t in (dQ, dK, dV)], 1)
    dx, rwq, rwk = S.qk_norm_rope_grad(x, *w, *tabs, p, Hq, EPS, inter, dY)
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + EPS)
    xh = np.abs(x * r)
    # |dz| of a pair is at most the sum of its two |dy|: twice the row's largest
    wmax = max(np.abs(w[0]).max(), np.abs(w[1]).max())
    u = 2 * np.abs(dY).max(-1, keepdims=True) * wmax
    _close(dqkv.reshape(B * N, H, d), dx, r * u * (1 + xh.max(-1, keepdims=True) * xh.mean(-1, keepdims=True)), "dqkv")
    assert np.array_equal(P.f64(dqkv).reshape(B * N, H, d)[:, Hq + Hkv:], dY[:, Hq + Hkv:])
    for got, ref, hs in ((dwq, rwq, slice(0, Hq)), (dwk, rwk, slice(Hq, Hq + Hkv))):
        sizes = (2 * np.abs(dY[:, hs]).max(-1, keepdims=True) * xh[:, hs]).sum((0, 1))
        assert got.dtype == torch.float32
        assert np.all(np.abs(P.f64(got) - ref) <= 2.0 ** -17 * sizes)


def test_gradient_of_many_tokens_sums_over_all_blocks():
    # enough rows for every block of the persistent kernel to take several; the plain
    # sum in fp64 on the device.  A lane adds ~70 terms one after the other
    B, N, Hq, Hkv, d = 2, 6001, 8, 2, 128
    g, qkv, wq, wk, cos, sin = _inputs(B, N, Hq, Hkv, d, 128, 0, seed=5)
    layer = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    dQ, dK, dV = _normal(g, B, Hq, N, d), _normal(g, B, Hkv, N, d), _normal(g, B, Hkv, N, d)
    dqkv, dwq, dwk = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, dQ, dK, dV, None, EPS, False)
    layer.close()
    c, s = cos[:N, None].double(), sin[:N, None].double()
    for part, dy, got in ((qkv[:, :, :Hq], dQ, dwq), (qkv[:, :, Hq:Hq + Hkv], dK, dwk)):
        x, y = part.double(), dy.transpose(1, 2).double()
        xh = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        a, b = y[..., :64], y[..., 64:]
        terms = torch.cat((a * c + b * s, b * c - a * s), -1) * xh
        assert bool(((got.double() - terms.sum((0, 1, 2))).abs() <= 2.0 ** -17 * terms.abs().sum((0, 1, 2))).all())


def test_non_finite_value_rows_and_zero_rows():
    # value rows only pass: their infinities and NaN reach nothing else; a zero row with
    # eps > 0 stays zero
    B, N, Hq, Hkv, d = 1, 9, 2, 1, 64
    g, qkv, wq, wk, cos, sin = _inputs(B, N, Hq, Hkv, d, 64, 0)
    qkv = qkv.clone()
    qkv[0, 3, 3] = float("nan")
    qkv[0, 4, 3] = float("inf")
    qkv[0, 5, 0] = 0
    layer = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    Q, K, V = layer.qk_norm_rope(qkv, wq, wk, cos, sin)
    assert bool(Q.isfinite().all()) and bool(K.isfinite().all()) and bool((Q[0, 0, 5] == 0).all())
    assert bool(V[0, 0, 3].isnan().all()) and bool(V[0, 0, 4].isinf().all())
    dV = _normal(g, 1, 1, N, d)
    dV[0, 0, 2] = float("nan")
    out = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, torch.ones_like(Q), torch.ones_like(K), dV)
    assert bool(out[0][:, :, :3].isfinite().all()) and bool(out[1].isfinite().all()) and bool(out[2].isfinite().all())
    assert bool(out[0][0, 2, 3].isnan().all())
    # eps = 0 takes the zero row's own outputs to NaN and nothing else
    out = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, torch.ones_like(Q), torch.ones_like(K), dV, eps=0.0)
    rows = out[0][0, :, :3].isfinite().all(-1)
    assert not bool(rows[5, 0]) and int(rows.sum()) == 3 * N - 1 and bool(out[2].isfinite().all())
    layer.close()


def test_positions_outside_the_tables_are_skipped():
    B, N, Hq, Hkv, d = 1, 6, 2, 1, 64
    g, qkv, wq, wk, cos, sin = _inputs(B, N, Hq, Hkv, d, 64, 0)
    layer = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    pos = torch.tensor([[0, 1, cos.shape[0], 3, -1, 5]], dtype=torch.int32, device=DEV)
    Q, K, V = (torch.full((1, h, N, d), 7.0, device=DEV, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    sas.sas_qk_norm_rope_fwd(layer.h, qkv, wq, wk, cos, sin, Q, K, V, pos)
    assert sas.sas_get_device_status(layer.h) == sas.SAS_ERR_INVALID_ARG
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    good = torch.tensor([[0, 1, 0, 3, 0, 5]], dtype=torch.int32, device=DEV)
    ref = layer.qk_norm_rope(qkv, wq, wk, cos, sin, good)
    for got, want in zip((Q, K, V), ref):
        assert torch.equal(got[:, :, [0, 1, 3, 5]], want[:, :, [0, 1, 3, 5]]) and bool((got[:, :, [2, 4]] == 7).all())
    dqkv = torch.full((1, N, 4, d), 7.0, device=DEV, dtype=torch.bfloat16)
    dw = torch.empty(2, d, device=DEV)
    sas.sas_qk_norm_rope_bwd(layer.h, qkv, wq, wk, cos, sin, *ref, dqkv, dw[0], dw[1], pos)
    assert sas.sas_get_device_status(layer.h) == sas.SAS_ERR_INVALID_ARG
    assert bool((dqkv[:, [2, 4]] == 7).all()) and bool(dw.isfinite().all())
    layer.close()


def test_refusals():
    B, N, Hq, Hkv, d = 1, 6, 2, 1, 64
    g, qkv, wq, wk, cos, sin = _inputs(B, N, Hq, Hkv, d, 64, 0)
    layer = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    good = (qkv, wq, wk, cos, sin)
    layer.qk_norm_rope(*good)
    before = sas.sas_launch_count(layer.h)
    with pytest.raises(sas.SasError, match="max_pos"):
        layer.qk_norm_rope(qkv, wq, wk, cos[:5], sin[:5])
    with pytest.raises(sas.SasError, match="rot"):
        layer.qk_norm_rope(qkv, wq, wk, *_tables(N, 24))
    with pytest.raises(sas.SasError, match="rot"):
        layer.qk_norm_rope(qkv, wq, wk, *_tables(N, 80))
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(sas.SasError, match="eps"):
            layer.qk_norm_rope(*good, eps=eps)
    with pytest.raises(sas.SasError, match="misaligned"):
        odd = torch.empty(qkv.numel() + 1, device=DEV, dtype=torch.bfloat16)[1:].view(qkv.shape)
        layer.qk_norm_rope(odd, wq, wk, cos, sin)
    with pytest.raises(sas.SasError, match="row stride"):
        wide = torch.empty(1, N, 4 * d + 4, device=DEV, dtype=torch.bfloat16)
        layer.qk_norm_rope(wide[:, :, :4 * d].unflatten(-1, (4, d)), wq, wk, cos, sin)
    with pytest.raises(ValueError, match="qkv"):
        layer.qk_norm_rope(qkv[:, :, :3], wq, wk, cos, sin)
    with pytest.raises(ValueError, match="contiguous"):
        layer.qk_norm_rope(qkv.transpose(2, 3).contiguous().transpose(2, 3), wq, wk, cos, sin)
    with pytest.raises(ValueError, match="wq"):
        layer.qk_norm_rope(qkv, wq.float(), wk, cos, sin)
    with pytest.raises(ValueError, match="dQ"):
        layer.qk_norm_rope_bwd(*good, qkv, qkv, qkv)
    dq, dk = torch.zeros(B, Hq, N, d, device=DEV, dtype=torch.bfloat16), torch.zeros(B, Hkv, N, d, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(sas.SasError, match="dqkv"):
        layer.qk_norm_rope_bwd(*good, dq, dk, dk, out=(qkv, torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)))
    assert sas.sas_launch_count(layer.h) == before
    layer.close()


# ------------------------------------------------------------------ into cache pages

@pytest.mark.parametrize("Hq,Hkv,d,rot,inter,pad", [(4, 2, 128, 128, False, 0), (8, 1, 64, 32, True, 16),
                                                    (3, 3, 64, 64, False, 0), (32, 4, 128, 64, True, 0)])
@pytest.mark.parametrize("T", [1, 7, 90])
def test_append_matches_the_oracle_and_leaves_the_rest(Hq, Hkv, d, rot, inter, pad, T):
    g, qkv, wq, wk, cos, sin = _inputs(1, T, Hq, Hkv, d, rot, pad, seed=T)
    qkv = qkv[0]
    pages = 5
    perm = torch.randperm(pages * 64, generator=g, device=DEV)[:T]
    slots = perm.to(torch.int64)
    positions = torch.randint(0, cos.shape[0], (T,), generator=g, device=DEV, dtype=torch.int32)
    if T > 1:
        slots[T // 2] = -1          # padding
        positions[T // 2] = -1
    Kc, Vc = _normal(g, pages, Hkv, 64, d), _normal(g, pages, Hkv, 64, d)
    K0, V0 = Kc.clone(), Vc.clone()
    ch = sas.SasChunk(T, Hq, Hkv, d, 8, pages, T)
    out = torch.full((T, Hq, d), 7.0, device=DEV, dtype=torch.bfloat16)
    Q = ch.append(qkv, wq, wk, cos, sin, positions, slots, Kc, Vc, EPS, inter, out=out)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()
    live = slots.cpu().numpy() >= 0
    x = P.f64(qkv)[live]
    w = (P.f64(wq), P.f64(wk))
    rq, rk, rv = S.qk_norm_rope(x, *w, P.f64(cos), P.f64(sin), positions.cpu().numpy()[live], Hq, EPS, inter)
    zmax = _row_scale(x, w, Hq)
    lt = torch.from_numpy(live).to(DEV)
    _close(Q[lt], rq, zmax[:, :Hq], "Q")
    assert bool((Q[~lt] == 7).all())
    at = (slots[lt] // 64, slice(None), slots[lt] % 64)
    _close(Kc[at], rk, zmax[:, Hq:Hq + Hkv], "K")
    assert np.array_equal(P.f64(Vc[at]), rv)
    Kc[at], Vc[at] = K0[at], V0[at]
    assert torch.equal(Kc, K0) and torch.equal(Vc, V0)


def test_append_skips_what_is_out_of_range():
    T, Hq, Hkv, d = 5, 2, 1, 64
    g, qkv, wq, wk, cos, sin = _inputs(1, T, Hq, Hkv, d, 64, 0)
    Kc = torch.zeros(2, Hkv, 64, d, device=DEV, dtype=torch.bfloat16)
    Vc = torch.zeros_like(Kc)
    ch = sas.SasChunk(4, Hq, Hkv, d, 2, 2, T)
    slots = torch.tensor([3, 128, -2, 5, 1 << 40], dtype=torch.int64, device=DEV)
    positions = torch.tensor([0, 1, 2, cos.shape[0], 4], dtype=torch.int32, device=DEV)
    out = torch.full((T, Hq, d), 7.0, device=DEV, dtype=torch.bfloat16)
    ch.append(qkv[0], wq, wk, cos, sin, positions, slots, Kc, Vc, out=out)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
    assert bool((out[1:] == 7).all()) and not bool((out[0] == 7).all())
    assert torch.equal(Vc[0, 0, 3], qkv[0, 0, 3])
    Vc[0, 0, 3] = 0
    assert bool((Vc == 0).all())
    with pytest.raises(sas.SasError, match="max_tokens"):
        ch.append(qkv[0].repeat(2, 1, 1), wq, wk, cos, sin, positions.repeat(2), slots.repeat(2), Kc, Vc)
    with pytest.raises(ValueError, match="K_cache"):
        ch.append(qkv[0], wq, wk, cos, sin, positions, slots, Kc[:1], Vc[:1])
    with pytest.raises(ValueError, match="slots"):
        ch.append(qkv[0], wq, wk, cos, sin, positions, slots.int(), Kc, Vc)
    ch.close()


def test_append_past_two_to_the_31_elements():
    # pages at the end of caches of 2.7e9 elements each
    pages, Hq, Hkv, d, T = 41000, 8, 8, 128, 3
    g, qkv, wq, wk, cos, sin = _inputs(1, T, Hq, Hkv, d, 128, 0)
    Kc = torch.empty(pages, Hkv, 64, d, device=DEV, dtype=torch.bfloat16)
    Vc = torch.empty_like(Kc)
    ch = sas.SasChunk(T, Hq, Hkv, d, 4, pages, T)
    slots = torch.tensor([pages * 64 - 1, 5, (pages - 7) * 64], dtype=torch.int64, device=DEV)
    positions = torch.arange(T, dtype=torch.int32, device=DEV)
    small = sas.SasChunk(T, Hq, Hkv, d, 4, 3, T)
    ks, vs = torch.empty(3, Hkv, 64, d, device=DEV, dtype=torch.bfloat16), torch.empty(3, Hkv, 64, d, device=DEV, dtype=torch.bfloat16)
    near = torch.tensor([63, 64 + 5, 128], dtype=torch.int64, device=DEV)
    Q = ch.append(qkv[0], wq, wk, cos, sin, positions, slots, Kc, Vc)
    Qs = small.append(qkv[0], wq, wk, cos, sin, positions, near, ks, vs)
    assert torch.equal(Q, Qs)
    for a, b in zip(slots.tolist(), near.tolist()):
        assert torch.equal(Kc[a // 64, :, a % 64], ks[b // 64, :, b % 64])
        assert torch.equal(Vc[a // 64, :, a % 64], vs[b // 64, :, b % 64])
    ch.close()
    small.close()


def test_caller_buffers_and_a_captured_step():
    # own outputs, on another stream, captured once and replayed on new inputs
    B, N, Hq, Hkv, d = 2, 50, 4, 2, 128
    g, qkv, wq, wk, cos, sin = _inputs(B, N, Hq, Hkv, d, 128, 0)
    layer = sas.SasLayer(B, Hq, N, d, 0, Hkv=Hkv)
    want = layer.qk_norm_rope(qkv, wq, wk, cos, sin)
    dy = tuple(_normal(g, *t.shape) for t in want)
    want += layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, *dy)
    fwd = tuple(torch.zeros_like(t) for t in want[:3])
    bwd = tuple(torch.zeros_like(t) for t in want[3:])
    side, x = torch.cuda.Stream(), torch.zeros_like(qkv)
    torch.cuda.synchronize()
    layer.qk_norm_rope(x, wq, wk, cos, sin, out=fwd, stream=side)       # sets the kernels' attributes
    layer.qk_norm_rope_bwd(x, wq, wk, cos, sin, *dy, out=bwd, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        assert layer.qk_norm_rope(x, wq, wk, cos, sin, out=fwd, stream=side) is fwd
        assert layer.qk_norm_rope_bwd(x, wq, wk, cos, sin, *dy, out=bwd, stream=side) is bwd
    for scale in (1, 2):
        x.copy_(qkv * scale)
        for t in fwd + bwd:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        ref = want if scale == 1 else layer.qk_norm_rope(x, wq, wk, cos, sin) + layer.qk_norm_rope_bwd(x, wq, wk, cos, sin, *dy)
        assert all(torch.equal(a, b) for a, b in zip(fwd + bwd, ref))
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    with pytest.raises(ValueError, match="Q must"):
        layer.qk_norm_rope(qkv, wq, wk, cos, sin, out=(fwd[1], fwd[1], fwd[2]))
    layer.close()
