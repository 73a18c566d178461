"""The entry points go by the sizes of their handle, not by those of the tensors they are given: tensors of other
sizes are refused before any address is taken.  No GPU: a handle's sizes are all that is looked at."""
import ctypes

import pytest
import torch

from paper_2609_13141_gb300 import sas

I32, BF = torch.int32, torch.bfloat16


@pytest.fixture
def chunk():
    h = sas._Handle()
    h.sizes = 4, 64, 8, (16, 2, 64, 64)    # 4 heads of 64, tables of 8 blocks, caches of 16 pages of 2 KV groups
    return h


def _ints(*shape):
    return torch.zeros(*shape, dtype=I32)


@pytest.mark.parametrize("table", [(2, 7), (2, 9), (1, 8), (16,), (2, 8, 1)])
def test_tables_of_other_sizes_are_refused(chunk, table):
    with pytest.raises(ValueError, match="block_table must have 2 rows and 8 columns"):
        sas.sas_chunk_attention(chunk, torch.zeros(3, 4, 64, dtype=BF), torch.zeros(16, 2, 64, 64, dtype=BF),
                                torch.zeros(16, 2, 64, 64, dtype=BF), _ints(*table), _ints(3), _ints(2),
                                torch.zeros(3, 4, 64, dtype=BF))
    with pytest.raises(ValueError, match="block_table must have 2 rows and 8 columns"):
        sas.sas_chunk_plan(chunk, _ints(2), _ints(2), _ints(5), _ints(1), _ints(*table), _ints(2), _ints(3), _ints(6),
                           torch.zeros(6, dtype=torch.int64), _ints(1))


@pytest.mark.parametrize("h", [None, ctypes.c_void_p()])
def test_handles_from_elsewhere_are_refused(h):
    with pytest.raises(sas.SasError, match="handle"):
        sas.sas_chunk_attention(h, torch.zeros(3, 4, 64, dtype=BF), None, None, _ints(2, 8), _ints(3), _ints(2), None)
    with pytest.raises(sas.SasError, match="handle"):
        sas.sas_qk_norm_rope_fwd(h, None, None, None, torch.zeros(4, 32), torch.zeros(4, 32), None, None, None)
