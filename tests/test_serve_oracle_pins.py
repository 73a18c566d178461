"""Pins of the serving-step oracle: hand examples, torch's own operators, differences."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_by_hand(inter):
    # a quarter turn of the first pair, the second unturned, the rest outside the rotation
    z = np.arange(1.0, 7.0)
    y = S.rotate(z, [0.0, 1.0], [1.0, 0.0], inter)
    want = [-2, 1, 3, 4, 5, 6] if inter else [-3, 2, 1, 4, 5, 6]
    assert np.array_equal(y, want)


@pytest.mark.parametrize("inter,rot", [(False, 8), (True, 8), (False, 4), (True, 4)])
def test_norm_rope_gradient_against_autograd_and_differences(inter, rot):
    rng = np.random.default_rng(rot)
    T, Hq, Hkv, d, eps = 3, 2, 1, 8, 1e-3
    qkv, dY = rng.normal(size=(T, Hq + 2 * Hkv, d)), rng.normal(size=(T, Hq + 2 * Hkv, d))
    wq, wk = rng.normal(size=d), rng.normal(size=d)
    ang = rng.normal(size=(5, rot // 2))
    cos, sin, pos = np.cos(ang), np.sin(ang), [4, 0, 2]

    def loss(qkv, wq, wk):
        return sum(float((a * b).sum()) for a, b in
                   zip(S.qk_norm_rope(qkv, wq, wk, cos, sin, pos, Hq, eps, inter), (dY[:, :Hq], dY[:, Hq:-Hkv], dY[:, -Hkv:])))

    dx, dwq, dwk = S.qk_norm_rope_grad(qkv, wq, wk, cos, sin, pos, Hq, eps, inter, dY)
    h = 1e-6
    for args, k, grad in (((qkv, wq, wk), 0, dx), ((qkv, wq, wk), 1, dwq), ((qkv, wq, wk), 2, dwk)):
        flat = args[k].reshape(-1)
        for i in range(0, flat.size, 3):
            keep = flat[i]
            flat[i] = keep + h
            up = loss(*args)
            flat[i] = keep - h
            down = loss(*args)
            flat[i] = keep
            # central differences of an O(10) function: error ~ h^2 + 1e-15 * 10 / h
            assert abs((up - down) / (2 * h) - grad.reshape(-1)[i]) < 1e-7
    # torch's rms_norm and complex products, with autograd
    x = torch.tensor(qkv, requires_grad=True)
    w = [torch.tensor(v, requires_grad=True) for v in (wq, wk)]
    ph = torch.polar(torch.ones(5, rot // 2, dtype=torch.float64), torch.tensor(ang))[pos][:, None]
    total = (x[:, -Hkv:] * torch.tensor(dY[:, -Hkv:])).sum()
    for part, wt, g in ((x[:, :Hq], w[0], dY[:, :Hq]), (x[:, Hq:-Hkv], w[1], dY[:, Hq:-Hkv])):
        z = torch.nn.functional.rms_norm(part, (d,), wt, eps)
        a, b = (z[..., 0:rot:2], z[..., 1:rot:2]) if inter else (z[..., :rot // 2], z[..., rot // 2:rot])
        y = torch.complex(a.contiguous(), b.contiguous()) * ph
        y = torch.stack((y.real, y.imag), -1).flatten(-2) if inter else torch.cat((y.real, y.imag), -1)
        total = total + (torch.cat((y, z[..., rot:]), -1) * torch.tensor(g)).sum()
    total.backward()
    assert abs(loss(qkv, wq, wk) - float(total.detach())) < 1e-10
    for got, want in ((dx, x.grad), (dwq, w[0].grad), (dwk, w[1].grad)):
        assert np.abs(got - want.numpy()).max() < 1e-11


def test_plan_by_hand():
    table = np.full((3, 3), -1)
    table[0, 0], table[2, :2] = 9, (7, 8)
    r = S.plan([63, 0, 128], [2, 0, 1], [4, 5, 6, 3], 1, table, 5)
    assert r[0] == [65, 0, 129] and r[1] == [0, 2, 2, 3] and r[2] == [63, 64, 128, -1, -1]
    assert r[3] == [9 * 64 + 63, 5 * 64, 6 * 64, -1, -1] and r[4] == 3
    assert r[5].tolist() == [[9, 5, -1], [-1, -1, -1], [7, 8, 6]]


def test_chunk_attention_is_sdpa_of_the_sequence():
    rng = np.random.default_rng(0)
    Hq, Hkv, d, P = 4, 2, 8, 6
    K, V = rng.normal(size=(P, Hkv, 64, d)), rng.normal(size=(P, Hkv, 64, d))
    table, cu, kv = np.array([[5, 2, 1], [0, -1, -1], [3, 4, -1]]), [0, 3, 3, 9], [150, 40, 70]
    Q = rng.normal(size=(9, Hq, d))
    O, LSE, A, _ = S.chunk_attention(Q, K, V, table, cu, kv, 0.3)
    for b in (0, 2):
        n, L = cu[b + 1] - cu[b], kv[b]
        pages = table[b][:-(-L // 64)]
        k, v = (torch.tensor(np.concatenate([c[p] for p in pages], 1)[:, :L]).repeat_interleave(2, 0) for c in (K, V))
        q = torch.tensor(Q[cu[b]:cu[b + 1]]).transpose(0, 1)
        mask = torch.arange(L) <= torch.arange(L - n, L)[:, None]
        for x, y in ((v, O), (v.abs(), A)):
            want = torch.nn.functional.scaled_dot_product_attention(q, k, x, attn_mask=mask, scale=0.3).transpose(0, 1)
            assert np.abs(y[cu[b]:cu[b + 1]] - want.numpy()).max() < 1e-12
        z = (q @ k.transpose(1, 2) * 0.3).masked_fill(~mask, -math.inf)
        assert np.abs(LSE[cu[b]:cu[b + 1]].T - torch.logsumexp(z, -1).numpy()).max() < 1e-12


def test_verify_by_hand():
    p = np.array([[.5, .5, 0], [.2, .3, .5], [.1, .1, .8]])
    q = np.array([[.25, .5, .25], [.6, .3, .1]])
    e = np.array([[1.0, 1.0, 1.0]])
    # 0.9 * 0.5 < 0.5: accepted; 0.4 * 0.6 < 0.2 fails: residual of row 1 is (0, 0, 0.4)
    a, t = S.verify([1, 0], [0, 2], p, q, np.array([.9, .4]), e, 2)
    assert a.tolist() == [1] and t.tolist() == [[1, 2, -1]]
    # both accepted: argmax p_2 / e
    a, t = S.verify([1, 0], [0, 2], p, q, np.array([.9, .3]), np.array([[.1, 1.0, 8.5]]), 2)
    assert a.tolist() == [2] and t.tolist() == [[1, 0, 0]]
    # certain drafts: accepted with probability p; the residual is p without the draft; ties go down
    a, t = S.verify([0, 0], [0, 2], p, None, np.array([.4, .3]), e, 2)
    assert a.tolist() == [1] and t.tolist() == [[0, 2, -1]]
    # an empty residual (p = q) falls back to p
    a, t = S.verify([2, 0], [0, 2], np.array([[.5, .5, 0]] * 3), np.array([[.5, .5, 0]] * 2), np.array([0., 0.]), e, 2)
    assert a.tolist() == [0] and t.tolist() == [[0, -1, -1]]


def test_verify_draws_from_the_target():
    # whatever the draft's distribution, the first token is distributed as p_0
    rng = np.random.default_rng(1)
    n, V = 40000, 4
    p, q = np.array([.1, .2, .3, .4]), np.array([.4, .3, .2, .1])
    x = rng.choice(V, size=n, p=q)
    target = np.repeat(p[None], 2 * n, 0)
    _, out = S.verify(x, list(range(n + 1)), target, np.repeat(q[None], n, 0), rng.random(n), rng.exponential(size=(n, V)), 1)
    freq = np.bincount(out[:, 0], minlength=V) / n
    assert np.all(np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / n))   # five standard deviations
