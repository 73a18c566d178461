"""Chunk attention over live keys that are not finite.

A row that sees a NaN score is NaN, however its unit is cut into splits, and so is its LSE; rows, heads and requests
that do not see one are as without it.  A row whose scores in a whole split are -inf gets nothing from there."""
import math

import pytest
import torch

from paper_2609_13141_gb300 import sas
from tests.test_gpu_chunk_attention import DEV, _case, _compare

pytestmark = pytest.mark.gpu


def _fill(cache, table, b, head, lo, hi, value):
    """Keys lo .. hi - 1 of request b, one KV head."""
    for p in range(lo // 64, -(-hi // 64)):
        cache[int(table[b, p]), head, max(lo - 64 * p, 0):min(hi - 64 * p, 64)] = value


# few rows and full tiles, units of a few and of many splits
SHAPES = [
    (4, 2, 128, [(3000, 1), (500, 3)]),
    (8, 2, 64, [(5000, 3), (700, 1)]),
    (8, 1, 128, [(19000, 1)]),                  # many splits a row: their shares are joined too
    (1, 2, 64, [(6000, 128), (90, 5)]),         # a full tile
    (4, 2, 128, [(4500, 33), (10, 40)]),
    (1, 1, 128, [(1200, 1)]),
]


@pytest.mark.parametrize("G,Hkv,d,lens", SHAPES)
@pytest.mark.parametrize("tail", [True, False])
def test_live_nan_keys_reach_every_row_that_sees_them(G, Hkv, d, lens, tail):
    # from every page on to the end, and up to every page: some of them begin and end where a split does, so that
    # splits hold NaN scores only or none
    Q, K, V, table, cu, kv = _case(lens, G * Hkv, Hkv, d, seed=G + d)
    n, L = lens[0][1], int(kv[0])
    ch = sas.SasChunk(len(lens), G * Hkv, Hkv, d, table.shape[1], K.shape[0], Q.shape[0])
    R, M = ch.attention(Q, K, V, table, cu, kv)
    _compare(R, M, Q, K, V, table, cu, kv, 1 / math.sqrt(d))
    for page in range(0, -(-(L - n) // 64)):
        bad = K.clone()
        _fill(bad, table, 0, 0, 64 * page if tail else 0, L if tail else min(64 * (page + 1), L - n), math.nan)
        O, LSE = ch.attention(Q, bad, V, table, cu, kv)
        assert bool(O[:n, :G].isnan().all()) and bool(LSE[:n, :G].isnan().all()), f"page {page}"
        O[:n, :G], LSE[:n, :G] = R[:n, :G], M[:n, :G]
        assert torch.equal(O, R) and torch.equal(LSE, M)      # everything else: as without them
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()


@pytest.mark.parametrize("G,Hkv,d,lens", SHAPES)
def test_scores_of_minus_infinity_count_for_nothing(G, Hkv, d, lens):
    Q, K, V, table, cu, kv = _case(lens, G * Hkv, Hkv, d, seed=G)
    Q = Q.abs() + 0.125
    context = lens[0][0]
    a, b = int(0.2 * context), int(0.9 * context)
    _fill(K, table, 0, 0, a, b, -math.inf)
    ch = sas.SasChunk(len(lens), G * Hkv, Hkv, d, table.shape[1], K.shape[0], Q.shape[0])
    O, LSE = ch.attention(Q, K, V, table, cu, kv)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()
    # in 64 bits, without those keys
    n, L = lens[0][1], int(kv[0])
    pages = table[0, :-(-L // 64)].long()
    keys, vals = (x[pages, 0].reshape(-1, d)[:L].double() for x in (K, V))
    seen = torch.ones(L, dtype=torch.bool, device=DEV)
    seen[a:b] = False
    z = torch.einsum("tgd,ld->tgl", Q[:n, :G].double(), keys.masked_fill(~seen[:, None], 0)) / math.sqrt(d)
    late = torch.arange(L, device=DEV) > (L - n + torch.arange(n, device=DEV))[:, None]
    z.masked_fill_((late | ~seen)[:, None], -math.inf)
    size = torch.einsum("tgd,ld->tgl", Q[:n, :G].double(), keys.masked_fill(~seen[:, None], 0).abs()).amax(-1) / math.sqrt(d)
    p = torch.softmax(z, -1)
    ref, A = p @ vals, p @ vals.abs()
    # the bounds of the finite cases: P and O in bf16, logits off by delta
    delta = (2.0 ** -17 * size)[..., None]
    assert bool(((O[:n, :G].double() - ref).abs() <= 2.0 ** -8 * (A + ref.abs()) + (2 * delta + 2.0 ** -16) * A).all())
    assert bool(((LSE[:n, :G].double() - torch.logsumexp(z, -1)).abs() <= delta[..., 0] + 2.0 ** -15).all())
