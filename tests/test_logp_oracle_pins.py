"""Pins of the log-probability oracle: hand values, torch, central differences."""
import math

import numpy as np
import pytest
import torch

from oracle import logp_oracle as L


def test_hand_values():
    lp, h, lse = L.row([0.0, math.log(3.0)], 1)
    assert lp == pytest.approx(math.log(0.75)) and lse == pytest.approx(math.log(4.0))
    assert h == pytest.approx(-(0.25 * math.log(0.25) + 0.75 * math.log(0.75)))
    assert L.row([2.0, -math.inf], 0) == (0.0, 0.0, 2.0)
    assert L.row([-math.inf] * 3, 0)[2] == -math.inf


def test_against_torch():
    g = torch.Generator().manual_seed(0)
    z = torch.randn(6, 50, generator=g, dtype=torch.float64) * 3
    ref = torch.log_softmax(z, -1)
    for t in range(6):
        lp, h, lse = L.row(z[t].numpy(), t)
        assert lp == pytest.approx(float(ref[t, t])) and lse == pytest.approx(float(torch.logsumexp(z[t], 0)))
        assert h == pytest.approx(float(torch.distributions.Categorical(logits=z[t]).entropy()))
        assert L.alternatives(z[t].numpy(), 5).tolist() == torch.topk(z[t], 5).indices.tolist()


def test_alternatives_of_equal_columns():
    assert L.alternatives([1.0, 2.0, 2.0, -0.0, 0.0], 5).tolist() == [1, 2, 0, 3, 4]
    assert L.alternatives([math.nan, 1.0, -math.inf], 3).tolist() == [1, 2, -1]


def test_gradient_is_the_differences():
    rng = np.random.default_rng(1)
    z, x, gl, gh = rng.normal(size=12) * 2, 4, 0.7, -0.3
    f = lambda y: gl * L.row(y, x)[0] + gh * L.row(y, x)[1]  # noqa: E731
    _, h, lse = L.row(z, x)
    g = L.row_grad(z, x, lse, h, gl, gh)
    for v in range(12):
        e = np.zeros(12)
        e[v] = 1e-5
        assert g[v] == pytest.approx((f(z + e) - f(z - e)) / 2e-5, abs=1e-8)
    masked = np.where(np.arange(12) == 7, -math.inf, z)
    _, h, lse = L.row(masked, x)
    assert L.row_grad(masked, x, lse, h, gl, gh)[7] == 0.0
