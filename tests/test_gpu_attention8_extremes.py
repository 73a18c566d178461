"""Attention over an 8-bit cache where the scales of pages or the sizes of queries are extreme: the scores' factor (query times
key scale) outside fp32's range, value scales of one request at either end of what the append writes.  Cases, plain form and
bounds are test_gpu_attention8's."""
import math

import pytest
import torch

from paper_2609_13141_gb300 import sas
from tests.test_gpu_attention8 import DEV, E4, I32, _case, _chunk, _compare, _plain

pytestmark = pytest.mark.gpu

# heads a KV head, requests: each of the kernels at its heights (8 and 16 rows a tile, one and two 128-row tiles a block), with
# pages of which rows see a part, requests of one token and requests of many splits
SHAPES = [(4, [(500, 1), (90, 1), (0, 1), (63, 1)]), (8, [(9000, 1)]), (2, [(500, 5), (3, 5), (700, 4)]), (1, [(7000, 16)]),
          (2, [(500, 30), (90, 9), (0, 1)]), (1, [(6000, 64)]), (4, [(700, 90), (3, 40), (64, 1)]), (1, [(4000, 300)])]


def _dead(case, head):
    """The keys of a request's last page and of every second one before it become zero, as a step on zeros leaves them."""
    K, sk, table = case[1], case[3], case[5]
    for p in (p for row in table.tolist() for p in [p for p in row if p >= 0][::-2]):
        x = K.view(torch.uint8)[p, head]
        x[(x & 0x7F) != 0x7F] = 0          # what no token sees stays NaN
        sk[p, head] = 2.0 ** -64


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,lens", SHAPES)
def test_zero_and_tiny_queries_over_zero_keys(G, lens, d):
    """A product of 0 between finite numbers is a score of 0, however small query and scale are."""
    case = _case(lens, 2 * G, 2, d, seed=G + d)
    Q = case[0]
    _dead(case, 0)
    _dead(case, 1)
    Q[:, 0] = 0
    Q[::2, G - 1] *= 2.0 ** -120
    Q[1::2, G] = 0
    ch = _chunk(case)
    O, LSE = ch.attention8(*case)
    _compare(O, LSE, case, 1 / math.sqrt(d))
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,new", [(4, [1, 1, 3]), (2, [70, 10, 33]), (4, [400, 130])])
def test_a_step_on_zeros(G, new, d):
    """append8 of zero rows, attention8 over what it wrote: zeros, and the logarithm of how many."""
    B, T = len(new), sum(new)
    table = torch.arange(8 * B, dtype=I32, device=DEV).view(B, 8)
    ch = sas.SasChunk(B, 2 * G, 2, d, 8, 8 * B, T)
    K, V = (torch.full((8 * B, 2, 64, d), 0x7F, dtype=torch.uint8, device=DEV).view(E4) for _ in range(2))
    sk, sv = (torch.full((8 * B, 2), math.nan, device=DEV) for _ in range(2))
    one, turn = torch.ones(d, device=DEV, dtype=torch.bfloat16), torch.rand(512, d // 2, device=DEV)
    n = torch.tensor(new, dtype=I32, device=DEV)
    pos = torch.cat([torch.arange(k, dtype=I32, device=DEV) for k in new])
    slots = torch.cat([table[b].long().repeat_interleave(64)[:k] * 64 + torch.arange(k, device=DEV) % 64 for b, k in enumerate(new)])
    cu = torch.cat([torch.zeros(1, dtype=I32, device=DEV), n.cumsum(0, dtype=I32)])
    Q = ch.append8(torch.zeros(T, 2 * G + 4, d, device=DEV, dtype=torch.bfloat16), one, one, turn.cos(), turn.sin(), pos, slots, K, V, sk, sv)
    assert (Q == 0).all()
    O, LSE = ch.attention8(Q, K, V, sk, sv, table, cu, n)
    assert (O == 0).all()
    assert ((LSE - (pos + 1).float().log()[:, None]).abs() < 2.0 ** -15).all()
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,lens", SHAPES)
def test_scores_below_the_least_number(G, lens, d):
    """A key whose score is under -2^128 has no weight; its page's other scores are 0, as its zero keys have it."""
    case = _case(lens, G, 1, d, seed=G + d, poison=False)
    Q, K, V, sk, sv, table, cu, kv = case
    K.view(torch.uint8).zero_()
    Q.zero_()
    Q[..., 3] = 2.0 ** 60
    first = table[:, 0].long()
    K.view(torch.uint8)[first, 0, 0, 3] = 0xB8          # -1
    sk[first] = 2.0 ** 100
    ch = _chunk(case)
    O, LSE = ch.attention8(*case)
    for b, L in enumerate(kv.tolist()):
        t0, t1 = int(cu[b]), int(cu[b + 1])
        pages = table[b, :-(-L // 64)].long()
        v = (V.view(torch.uint8)[pages, 0].view(E4).double() * sv[pages, 0].double()[:, None, None]).reshape(-1, d)[:L]
        for t in range(t0, t1):
            n = L - t1 + t      # keys but the first one
            if n == 0:
                continue        # a row of such a key alone: its largest score is -infinity in fp32
            # uniform weights: fp16 sums of 1 are exact, fp32 sums and the output's rounding are left
            ref, size = v[1:n + 1].mean(0), v[1:n + 1].abs().mean(0)
            assert ((O[t].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -16 * size).all(), t
            assert (LSE[t] - math.log(n)).abs().max() < 2.0 ** -15
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


def _values(case, logs, dead=()):
    """Scales 2^logs[i] for a request's i-th page of values, over and over; codes of pages from 2^100 on are small, so that
    their numbers are finite; pages i of `dead` hold zeros."""
    V, sv, table = case[2], case[4], case[5]
    for row in table.tolist():
        for i, p in enumerate([p for p in row if p >= 0]):
            k = i % len(logs)
            if logs[k] > 100:
                V[p] = (V[p].float() / 64).to(E4)
            if k in dead:
                V.view(torch.uint8)[p] = 0
            sv[p] = 2.0 ** logs[k]


FAR = [((60, -64), (1,)), ((120, -8, -64, -64), (2, 3)), ((-8, 120, -8), ()), ((120, -126, 60), ()), ((-64, 120, -64, 100, -64), (0, 2, 4)),
       ((120, 120, 119), ()), ((110, 75, 40, 5, -30, -65, -100), ()), ((120, 85, 50, 15, -20, -55, -64), (6,)), ((120, -8), (0,)), ((-126, -64), ())]


@pytest.mark.parametrize("logs,dead", FAR)
@pytest.mark.parametrize("G,lens,d", [(4, [(500, 1), (90, 1)], 128), (8, [(9000, 1)], 64), (2, [(700, 5)], 128), (2, [(500, 30), (90, 9)], 64),
                                      (1, [(6000, 64)], 128), (4, [(700, 90)], 128), (1, [(4000, 300)], 128), (1, [(4000, 300)], 64), (2, [(2500, 1)] * 200, 64)])
def test_value_scales_at_the_ends_of_their_range(G, lens, d, logs, dead):
    """What a row's output may be off by is in units of its largest values: 2^-25 of them a key (times the spread 64 within which
    pages share a unit), where its weights are rounded to fp16."""
    case = _case(lens, G, 1, d, seed=G + d, poison=False)
    _values(case, logs, dead)
    ch = _chunk(case)
    O, LSE = ch.attention8(*case)
    ref, lse, A, size, U = _plain(*case, 1 / math.sqrt(d))
    assert (ref.abs() < 2.0 ** 127).all()
    delta = 2.0 ** -17 * size
    # the least bf16 number's half, too
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2.0 ** -16 + 2 * delta[..., None]) * A + 2.0 ** -25 * 64 * U.amax(-1, keepdim=True) + 2.0 ** -134
    assert O.isfinite().all()
    assert ((O.double() - ref).abs() <= tol).all(), float(((O.double() - ref).abs() / tol).max())
    assert ((LSE.double() - lse).abs() <= delta + 2.0 ** -15).all()
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


@pytest.mark.parametrize("G,lens,d", [(4, [(500, 1), (90, 1)], 128), (8, [(9000, 1)], 64), (2, [(700, 5)], 128), (2, [(500, 30)], 64), (4, [(700, 90)], 128),
                                      (1, [(4000, 300)], 128), (2, [(2500, 1)] * 200, 64), (1, [(2500, 2)] * 100, 128)])
def test_zero_values_under_any_scale_change_nothing_but_weights(G, lens, d):
    """Pages of zero values under scales of either end, among ordinary ones: to the precision of the ordinary ones' values."""
    case = _case(lens, G, 1, d, seed=G + d, poison=False)
    V, sv, table = case[2], case[4], case[5]
    for row in table.tolist():
        for i, p in enumerate([p for p in row if p >= 0]):
            if i % 3 != 1:
                V.view(torch.uint8)[p] = 0
                sv[p] = 2.0 ** (120 if i % 3 == 0 else -64)
    ch = _chunk(case)
    O, LSE = ch.attention8(*case)
    ref, lse, A, size, U = _plain(*case, 1 / math.sqrt(d))
    delta = 2.0 ** -17 * size
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2.0 ** -16 + 2 * delta[..., None]) * A + 2.0 ** -25 * 64 * U
    assert O.isfinite().all() and ((O.double() - ref).abs() <= tol).all()
    assert ((LSE.double() - lse).abs() <= delta + 2.0 ** -15).all()
