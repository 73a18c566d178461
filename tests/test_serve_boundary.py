"""Host-side checks of the serving-step entry points that need no GPU."""
import ctypes
import math

import pytest
import torch

from paper_2609_13141_gb300 import _build, sas


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return sas.lib()


@pytest.mark.parametrize("kw,expect", [
    (dict(max_seqs=0), sas.SAS_ERR_INVALID_ARG),
    (dict(max_seqs=8193), sas.SAS_ERR_UNSUPPORTED),
    (dict(Hq=12, Hkv=8), sas.SAS_ERR_INVALID_ARG),
    (dict(Hq=6, Hkv=2), sas.SAS_ERR_UNSUPPORTED),
    (dict(Hkv=0), sas.SAS_ERR_INVALID_ARG),
    (dict(Hq=131072, Hkv=65536), sas.SAS_ERR_UNSUPPORTED),
    (dict(d=96), sas.SAS_ERR_UNSUPPORTED),
    (dict(block=32), sas.SAS_ERR_UNSUPPORTED),
    (dict(max_blocks=0), sas.SAS_ERR_INVALID_ARG),
    (dict(max_blocks=32769), sas.SAS_ERR_UNSUPPORTED),
    (dict(num_pages=0), sas.SAS_ERR_INVALID_ARG),
    (dict(num_pages=1 << 30), sas.SAS_ERR_UNSUPPORTED),          # pages x KV heads past 31 bits
    (dict(max_tokens=0), sas.SAS_ERR_INVALID_ARG),
    (dict(max_tokens=(1 << 26) + 1), sas.SAS_ERR_UNSUPPORTED),
    (dict(sm_scale=-1.0), sas.SAS_ERR_INVALID_ARG),
    (dict(sm_scale=math.inf), sas.SAS_ERR_INVALID_ARG),
])
def test_chunk_create_rejects_bad_configs(lib, kw, expect):
    good = dict(max_seqs=4, Hq=8, Hkv=2, d=128, max_blocks=16, num_pages=32, max_tokens=64)
    assert sas.sas_chunk_create_status(**{**good, **kw}) == expect


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-GPU path")
def test_chunk_create_without_gpu_fails_cleanly(lib):
    st = sas.sas_chunk_create_status(max_seqs=4, Hq=8, Hkv=2, d=128, max_blocks=16, num_pages=32, max_tokens=64)
    assert st in (sas.SAS_ERR_CUDA, sas.SAS_ERR_UNSUPPORTED)


def test_serving_null_handles(lib):
    null, rope = ctypes.c_void_p(), sas.SasRopeConfig(64, 0, 8, 1e-6)
    assert lib.sas_chunk_plan(null, 1, 1, None, None, None, None, 0, *([None] * 8)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_chunk_append(null, rope, 1, None, 64, *([None] * 10)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_chunk_attention(null, 1, 1, *([None] * 9)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_chunk_verify(null, 1, 0, 0, 8, None, None, None, 8, None, 8, None, None, 8, None, None, None) == \
        sas.SAS_ERR_INVALID_ARG
    assert lib.sas_qk_norm_rope_fwd(null, rope, None, 64, *([None] * 9)) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_qk_norm_rope_bwd(null, rope, None, 64, *([None] * 9), 64, None, None, None) == sas.SAS_ERR_INVALID_ARG
    assert lib.sas_chunk_launch_count(null) == 0
    assert lib.sas_chunk_last_error(null) == b""
    lib.sas_chunk_destroy(null)   # no-op
