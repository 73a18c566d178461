"""Few tokens, whose launch has warps without any: slots and positions are views into longer arrays, at any
alignment their types allow, and what stands behind them changes nothing."""
import pytest
import torch

from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 1, 64), (8, 2, 128), (32, 8, 128), (1, 1, 64)])
@pytest.mark.parametrize("T", [1, 2, 3, 9])
def test_entries_behind_the_last_token_are_not_tokens(Hq, Hkv, d, T):
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    pages, H = 4, Hq + 2 * Hkv
    qkv = torch.randn(T, H, d, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.ones(d, device=DEV, dtype=torch.bfloat16)
    cos, sin = torch.ones(16, d // 2, device=DEV), torch.zeros(16, d // 2, device=DEV)
    slots = torch.randperm(pages * 64, generator=g, device=DEV)[:T + 9].to(torch.int64)
    pos = torch.arange(T + 9, device=DEV, dtype=torch.int32) % 16
    ch = sas.SasChunk(T, Hq, Hkv, d, 4, pages, T)
    got = []
    for tail in (slots, torch.full_like(slots, -1)):
        a, p = torch.empty(T + 10, dtype=torch.int64, device=DEV)[1:], torch.empty(T + 10, dtype=torch.int32, device=DEV)[1:]
        a.copy_(tail)
        p.copy_(pos)
        a[:T] = slots[:T]
        K, V = torch.zeros(2, pages, Hkv, 64, d, device=DEV, dtype=torch.bfloat16)
        Q = ch.append(qkv, w, w, cos, sin, p[:T], a[:T], K, V)
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
        at = (slots[:T] // 64, slice(None), slots[:T] % 64)
        assert torch.equal(V[at], qkv[:, Hq + Hkv:])
        V[at] = 0
        assert not bool(V.any())
        got.append((Q, K))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    ch.close()
