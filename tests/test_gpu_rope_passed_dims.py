"""Dims past the rotation pass alone: what is not finite in one of them does not reach another."""
import math

import pytest
import torch

from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N = 20


def _inputs(Hq, Hkv, d, rot):
    g = torch.Generator(device=DEV)
    g.manual_seed(d + rot)
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    ang = torch.rand(N, rot // 2, generator=g, device=DEV) * 6
    return normal(1, N, Hq + 2 * Hkv, d), normal(d), normal(d), ang.cos().contiguous(), ang.sin().contiguous(), normal


SHAPES = [(4, 2, 128, 64), (2, 2, 64, 16), (3, 3, 64, 32), (4, 1, 128, 112)]


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", SHAPES)
def test_a_weight_that_is_not_finite_keeps_to_its_dim(Hq, Hkv, d, rot, inter, value):
    qkv, wq, wk, cos, sin, normal = _inputs(Hq, Hkv, d, rot)
    layer = sas.SasLayer(1, Hq, N, d, 0, Hkv=Hkv)
    want = layer.qk_norm_rope(qkv, wq, wk, cos, sin, interleaved=inter)
    for at in (rot, rot + 5, d - 1):
        bad = wq.clone()
        bad[at] = value
        Q, K, V = layer.qk_norm_rope(qkv, bad, wk, cos, sin, interleaved=inter)
        assert not bool(Q[..., at].isfinite().any())
        Q[..., at] = want[0][..., at]
        assert torch.equal(Q, want[0]) and torch.equal(K, want[1]) and torch.equal(V, want[2])
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    layer.close()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", SHAPES)
def test_an_infinite_gradient_keeps_to_its_dim_of_dw(Hq, Hkv, d, rot, inter):
    # its row of dqkv has a mean over all dims and is not finite; the sums over tokens of the other dims are
    qkv, wq, wk, cos, sin, normal = _inputs(Hq, Hkv, d, rot)
    layer = sas.SasLayer(1, Hq, N, d, 0, Hkv=Hkv)
    dQ, dK, dV = normal(1, Hq, N, d), normal(1, Hkv, N, d), normal(1, Hkv, N, d)
    want = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, dQ, dK, dV, interleaved=inter)
    for at in (rot, rot + 5, d - 1):
        bad = dQ.clone()
        bad[0, Hq - 1, 7, at] = math.inf
        dqkv, dwq, dwk = layer.qk_norm_rope_bwd(qkv, wq, wk, cos, sin, bad, dK, dV, interleaved=inter)
        assert bool(dwq[at].isinf()) and not bool(dqkv[0, 7, Hq - 1].isfinite().any())
        dwq[at], dqkv[0, 7, Hq - 1] = want[1][at], want[0][0, 7, Hq - 1]
        assert torch.equal(dwq, want[1]) and torch.equal(dwk, want[2]) and torch.equal(dqkv, want[0])
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    layer.close()
