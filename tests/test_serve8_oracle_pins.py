"""Pins of the 8-bit cache's oracle, and refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import _build, sas


def test_e4m3_rounding_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = codes[torch.isfinite(codes)]
    assert (S.round_e4m3(codes.numpy()) == codes.numpy()).all()
    x = torch.cat([codes, (codes[:-1] + codes[1:]) / 2, torch.linspace(-448, 448, 4001, dtype=torch.float64),
                   torch.linspace(-0.02, 0.02, 4001, dtype=torch.float64)])
    want = x.float().to(torch.float8_e4m3fn).double().numpy()
    assert (S.round_e4m3(x.float().double().numpy()) == want).all()
    assert np.isnan(S.round_e4m3([math.inf, -math.inf, math.nan])).all()


@pytest.mark.parametrize("amax,k", [(448.0, 0), (448.0000001, 1), (3.5, -7), (3.5000001, -6), (0.0, -64), (1e-30, -64), (2.0 ** 100, 92),
                                    (3.3895e38, 120), (1.0, -8), (1.75, -8), (1.76, -7)])
def test_page_scale(amax, k):
    assert S.page_scale(amax) == 2.0 ** k


def test_append8_by_hand():
    """d = 16 of ones: the norm leaves 1, the rotation by 0 passes; a fresh page, then a larger value in a held one."""
    d, one = 16, np.ones(16)
    cos, sin = np.ones((4, 8)), np.zeros((4, 8))
    qkv = np.ones((2, 3, d))
    qkv[1, 2] = 1000.0
    K, V = np.full((2, 1, 64, d), 2.0), np.full((2, 1, 64, d), 2.0)
    Q, K2, V2, sk, sv = S.append8(qkv, one, one, cos, sin, [0, 1], [64, 5], 1, 0.0, False, K, V, np.full((2, 1), 0.5), np.full((2, 1), 0.5))
    assert (Q == 1).all() and sk.tolist() == [[0.5], [2.0 ** -8]] and sv.tolist() == [[4.0], [2.0 ** -8]]
    assert (K2[1, 0, 0] == 256).all() and (K2[1, 0, 1:] == 2).all()      # a fresh page: its other rows are left alone
    assert (K2[0, 0, 5] == 2).all() and (K2[0, 0, 4] == 2).all()          # the scale stays
    assert (V2[0, 0, 5] == 250).all() and (V2[0, 0, 4] == 0.25).all()     # it grows by 8


def test_null_handles_of_the_8_bit_entry_points():
    _build.build()
    lib, null, rope = sas.lib(), ctypes.c_void_p(), sas.SasRopeConfig(64, 0, 8, 1e-6)
    assert lib.sas_chunk_append8(null, rope, 1, None, 64, *([None] * 12)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_chunk_attention8(null, 1, 1, *([None] * 11)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_chunk_logprobs(null, 1, 8, None, 0, 8, None, 0, *([None] * 6)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_token_logprobs(null, 1, 8, None, 0, 8, *([None] * 5)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_token_logprobs_bwd(null, 1, 8, None, 0, 8, *([None] * 6), 8, None) == sas.SAS_ERR_INVALID_ARG
    assert {"sas_chunk_append8", "sas_chunk_attention8"} <= set(sas.header_functions())
