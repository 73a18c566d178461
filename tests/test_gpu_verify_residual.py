"""What follows a rejected draft: the residual max(p - q, 0) wherever it has a positive column, the target only
where it has none."""
import math

import pytest
import torch

from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


def _rejected(V, pad=0):
    """One request, one draft (column 3, target probability 0), the target below the draft everywhere."""
    wide = torch.full((4, V + pad), 1e-6, device=DEV)
    p, q, e = wide[:2, :V], wide[2:3, :V], torch.ones(1, V + pad, device=DEV)[:, :V]
    q.fill_(2e-6)
    q[0, 3], p[0, 3] = 0.5, 0.0
    q[0, V - 2], p[0, V - 2] = 0.5, 0.4        # the target's likeliest
    return p, q, e


def _next(p, q, e, certain=False):
    ch = sas.SasChunk(1, 1, 1, 64, 1, 1, 1)
    a, out = ch.verify(torch.tensor([3], dtype=I32, device=DEV), torch.tensor([0, 1], dtype=I32, device=DEV), p,
                       None if certain else q, torch.tensor([0.5], device=DEV), e, 1)
    st = sas.sas_chunk_get_device_status(ch.h)
    again = ch.verify(torch.tensor([3], dtype=I32, device=DEV), torch.tensor([0, 1], dtype=I32, device=DEV), p,
                      None if certain else q, torch.tensor([0.5], device=DEV), e, 1)
    assert torch.equal(again[1], out) and sas.sas_chunk_get_device_status(ch.h) == st
    ch.close()
    assert a.tolist() == [0] and int(out[0, 1]) == -1
    return int(out[0, 0]), st


# one block and many; rows that are read 16 bytes at a time and not
SIZES = [(7, 0), (32, 0), (1000, 3), (151936, 0), (151935, 2)]


@pytest.mark.parametrize("V,pad", SIZES)
@pytest.mark.parametrize("noise", [0.0, -1.0, math.nan])
def test_a_residual_without_usable_noise_gives_no_token(V, pad, noise):
    # the residual is positive in one column only, whose noise cannot be divided by: no column is left to choose,
    # least of all from the target, which would give the rejected draft or any other token the residual excludes
    for at in (0, V // 2, V - 1):
        if at == 3 or at == V - 2:
            continue
        p, q, e = _rejected(V, pad)
        p[0, at] = 3e-6
        e[0, at] = noise
        assert _next(p, q, e) == (-1, sas.SAS_ERR_INVALID_ARG)


@pytest.mark.parametrize("V,pad", SIZES)
def test_a_residual_too_small_for_its_noise_is_still_the_residual(V, pad):
    # 1e-44 / 50 is zero in 32 bits
    for at in (0, V // 2, V - 1):
        if at == 3 or at == V - 2:
            continue
        p, q, e = _rejected(V, pad)
        p[0, at], q[0, at], e[0, at] = 1e-44, 0.0, 50.0
        assert _next(p, q, e) == (at, sas.SAS_OK)
        e[0, at] = math.inf
        assert _next(p, q, e) == (at, sas.SAS_OK)


@pytest.mark.parametrize("V,pad", SIZES)
def test_an_empty_residual_takes_the_target(V, pad):
    p, q, e = _rejected(V, pad)
    assert _next(p, q, e) == (V - 2, sas.SAS_OK)
    e[0, V - 2] = 0.0        # of the target's columns the best whose noise is positive: equal ones, the lowest
    assert _next(p, q, e) == (0, sas.SAS_OK)


@pytest.mark.parametrize("V,pad", SIZES)
def test_a_certain_draft_leaves_the_other_columns(V, pad):
    p, q, e = _rejected(V, pad)
    p[0, 3] = 0.25           # u = 0.5: rejected, and no candidate any more
    assert _next(p, q, e, certain=True) == (V - 2, sas.SAS_OK)
    p[0] = 0
    p[0, 3], e[0, 3] = 0.25, 1.0   # nothing else has weight: the target itself
    assert _next(p, q, e, certain=True) == (3, sas.SAS_OK)
