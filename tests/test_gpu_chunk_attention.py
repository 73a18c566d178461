"""GPU parity of the chunk attention over a paged cache against the fp64 oracle.

Bounds, element by element.  P and O are rounded to bf16 (2^-8 each, of the terms
p_j |v_j| and of O); a logit is an fp32 sum of d products, off by at most delta =
2^-17 scale sum|q||k|, which moves O by 2 delta A with A the output on |V|, and the
fp32 sums add 2^-16 A.  LSE moves by delta, and by 2^-15 for the sums over the keys."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas
from tests import parity as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


def _case(lens, Hq, Hkv, d, seed=0, spare=2, poison=True, std=1.0):
    """lens: (cached, new) of each sequence.  Everything a token must not see is NaN or infinite."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    total = [c + n for c, n in lens]
    need = [-(-t // 64) for t in total]
    pages, width = sum(need) + spare, max(max(need), 1) + 1
    perm = torch.randperm(pages, generator=g, device=DEV).to(I32)
    table = torch.full((len(lens), width), -1, dtype=I32, device=DEV)
    K = torch.randn(pages, Hkv, 64, d, generator=g, device=DEV).to(torch.bfloat16)
    V = torch.randn(pages, Hkv, 64, d, generator=g, device=DEV).to(torch.bfloat16)
    k = 0
    for b, c in enumerate(need):
        table[b, :c] = perm[k:k + c]
        k += c
        if poison and total[b] % 64:
            last = int(perm[k - 1])
            K[last, :, total[b] % 64:] = float("nan")
            V[last, :, total[b] % 64:] = float("nan") if b % 2 else float("inf")
    if poison:
        for x in perm[k:].tolist():
            K[x], V[x] = float("nan"), float("nan")
    cu = torch.tensor([0] + np.cumsum([n for _, n in lens]).tolist(), dtype=I32, device=DEV)
    Q = (torch.randn(int(cu[-1]), Hq, d, generator=g, device=DEV) * std).to(torch.bfloat16)
    return Q, K, V, table, cu, torch.tensor(total, dtype=I32, device=DEV)


def _compare(O, LSE, Q, K, V, table, cu, kv, scale, rows=None):
    clean = lambda t: np.nan_to_num(P.f64(t), nan=0.0, posinf=0.0, neginf=0.0)  # noqa: E731
    ref, lse, A, S1 = S.chunk_attention(P.f64(Q), clean(K), clean(V), table.cpu().numpy(), cu.tolist(), kv.tolist(), scale)
    got = P.f64(O)
    live = ~np.isnan(lse)
    delta = (2.0 ** -17 * scale * S1)[..., None]
    tol = 2.0 ** -8 * (A + np.abs(ref)) + (2 * delta + 2.0 ** -16) * A
    err = np.abs(got - ref)
    assert np.isfinite(got[live]).all()
    assert np.all(err[live] <= tol[live]), f"O: worst {np.max(err[live] - tol[live]):.3g} over the bound"
    if LSE is not None:
        e = np.abs(P.f64(LSE) - lse)
        assert np.all(e[live] <= (delta[..., 0] + 2.0 ** -15)[live]), f"LSE off by {e[live].max():.3g}"


def _run(lens, Hq, Hkv, d, seed=0, scale=0.0, std=1.0):
    case = _case(lens, Hq, Hkv, d, seed, std=std)
    Q, K, V, table, cu, kv = case
    ch = sas.SasChunk(len(lens), Hq, Hkv, d, table.shape[1], K.shape[0], max(Q.shape[0], 1), scale)
    O, LSE = ch.attention(Q, K, V, table, cu, kv)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    O2, LSE2 = ch.attention(Q, K, V, table, cu, kv)
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2)   # equal inputs, equal bits, split or not
    ch.close()
    _compare(O, LSE, *case, scale or 1 / math.sqrt(d))


@pytest.mark.parametrize("G,d", [(1, 64), (2, 128), (4, 128), (8, 64), (1, 128), (4, 64), (8, 128), (2, 64)])
def test_lengths_that_meet_every_edge(G, d):
    # first tokens, page boundaries on either side, chunks shorter and longer than a tile, a sequence
    # without new tokens and one without any
    lens = [(0, 1), (0, 63), (0, 64), (0, 65), (63, 1), (64, 1), (65, 2), (127, 129), (200, 0), (0, 0), (31, 130), (300, 17)]
    _run(lens, 2 * G, 2, d, seed=G + d)


@pytest.mark.parametrize("G,Hkv,d,lens", [
    (4, 2, 128, [(3000, 1)]),                       # one token, the pages split over many items
    (8, 1, 64, [(5000, 3), (10, 1)]),
    (1, 3, 128, [(2000, 40)]),                      # a tile of 40 rows, the early ones blind to the last pages
    (2, 1, 64, [(700, 128), (1, 1), (64, 64)]),
    (4, 8, 128, [(1500, 5)] * 3),                   # drafted tokens
    (1, 1, 64, [(0, 700)]),                         # a prompt from nothing
    (4, 2, 128, [(64 * k + 7, 1 + 5 * k) for k in range(20)]),
])
def test_splits_and_mixed_batches(G, Hkv, d, lens):
    _run(lens, G * Hkv, Hkv, d, seed=len(lens))


@pytest.mark.parametrize("G,Hkv,d,lens", [
    (8, 1, 128, [(19000, 1)]),                      # one unit of long splits, few rows: all its blocks join it
    (1, 1, 64, [(6000, 128)]),                      # a full tile, rows blind to the last splits
    (4, 1, 128, [(4500, 33)]),                      # a full tile and one of four rows
    (1, 1, 128, [(600, 1)]),                        # one row in two or three splits
    (2, 2, 64, [(9000, 7), (300, 1)]),
    (1, 2, 128, [(2500, 70), (2500, 3)]),
])
def test_units_of_many_splits(G, Hkv, d, lens):
    _run(lens, G * Hkv, Hkv, d, seed=2 * len(lens) + G)


def test_scale_and_peaked_rows():
    # logits of +-100: the running maximum moves far and often
    _run([(500, 30), (90, 1)], 4, 2, 128, seed=3, scale=0.9, std=4.0)


def test_many_sequences():
    rng = np.random.default_rng(7)
    lens = [(int(c), int(n)) for c, n in zip(rng.integers(0, 90, 1500), rng.integers(0, 3, 1500))]
    _run(lens, 2, 1, 64, seed=1)


def test_rows_past_the_end_and_lse_none_are_left_alone():
    Q, K, V, table, cu, kv = _case([(100, 5), (3, 2)], 4, 2, 64)
    ch = sas.SasChunk(2, 4, 2, 64, table.shape[1], K.shape[0], 16)
    wide = torch.full((16, 4, 64), float("nan"), device=DEV, dtype=torch.bfloat16)
    wide[:7] = Q
    O = torch.full_like(wide, 7.0)
    LSE = torch.full((16, 4), 7.0, device=DEV)
    ch.attention(wide, K, V, table, cu, kv, out=(O, LSE))
    assert bool((O[7:] == 7).all()) and bool((LSE[7:] == 7).all())
    O2 = torch.full_like(wide, 7.0)
    ch.attention(wide, K, V, table, cu, kv, out=(O2, None))
    assert torch.equal(O, O2)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()
    _compare(O[:7], LSE[:7], Q, K, V, table, cu, kv, 1 / 8)


def test_chunks_of_a_prompt_give_the_prompt():
    # the same 400-token prompt in one chunk and in uneven ones: row by row the same keys
    Q, K, V, table, cu, kv = _case([(0, 400)], 8, 2, 128)
    ch = sas.SasChunk(1, 8, 2, 128, table.shape[1], K.shape[0], 400)
    whole, lse = ch.attention(Q, K, V, table, cu, kv)
    at = 0
    for n in (1, 63, 100, 7, 229):
        O, L = ch.attention(Q[at:at + n], K, V, table, torch.tensor([0, n], dtype=I32, device=DEV),
                            torch.tensor([at + n], dtype=I32, device=DEV))
        # two results within the bound of the same value; |V| ~ 1 gives A < 1.1, |O| <= A
        assert float((O.float() - whole[at:at + n].float()).abs().max()) <= 2 * (2.0 ** -8 * 4.4 + 2.0 ** -10)
        assert float((L - lse[at:at + n]).abs().max()) <= 2.0 ** -12
        at += n
    ch.close()


def test_one_token_agrees_with_the_decode_step():
    # a dense decode step and a chunk of one token read the same cache
    lens = [(4096, 1), (70, 1), (0, 1), (63, 1)]
    Q, K, V, table, cu, kv = _case(lens, 8, 2, 128, poison=False)
    ch = sas.SasChunk(4, 8, 2, 128, table.shape[1], K.shape[0], 4)
    O, LSE = ch.attention(Q, K, V, table, cu, kv)
    dec = sas.SasDecoder(4, 8, 2, 128, 0, table.shape[1], K.shape[0], dense=True)
    O2, LSE2, _ = dec.step(Q, K, V, table, kv)
    assert float((O.float() - O2.float()).abs().max()) <= 2 * (2.0 ** -8 * 4.4 + 2.0 ** -10)
    assert float((LSE - LSE2).abs().max()) <= 2.0 ** -12
    ch.close()
    dec.close()


def test_pages_past_two_to_the_31_elements():
    pages, Hq, Hkv, d = 41000, 8, 8, 128
    Q, K, V, table, cu, kv = _case([(130, 3)], Hq, Hkv, d, poison=False)
    big = torch.empty(2, pages, Hkv, 64, d, device=DEV, dtype=torch.bfloat16)
    far = torch.tensor([[pages - 1, 4, pages - 9, -1]], dtype=I32, device=DEV)
    for i in range(3):
        big[0, int(far[0, i])], big[1, int(far[0, i])] = K[int(table[0, i])], V[int(table[0, i])]
    a = sas.SasChunk(1, Hq, Hkv, d, 4, K.shape[0], 3)
    b = sas.SasChunk(1, Hq, Hkv, d, 4, pages, 3)
    x, y = a.attention(Q, K, V, table, cu, kv), b.attention(Q, big[0], big[1], far, cu, kv)
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    a.close()
    b.close()


def test_replayed_graph_follows_the_lengths_on_another_stream():
    lens = [(500, 9), (64, 1), (0, 40)]
    Q, K, V, table, cu, kv = _case(lens, 4, 1, 64, poison=False)
    ch = sas.SasChunk(3, 4, 1, 64, table.shape[1], K.shape[0], 50)
    out = (torch.empty_like(Q), torch.empty(Q.shape[:2], device=DEV))
    cu2, kv2 = torch.zeros_like(cu), torch.zeros_like(kv)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ch.attention(Q, K, V, table, cu2, kv2, out=out, stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ch.attention(Q, K, V, table, cu2, kv2, out=out, stream=side)
    for c, k in ((cu, kv), (torch.tensor([0, 1, 2, 30], dtype=I32, device=DEV), torch.tensor([509, 3, 40], dtype=I32, device=DEV))):
        cu2.copy_(c)
        kv2.copy_(k)
        g.replay()
        torch.cuda.synchronize()
        want = ch.attention(Q, K, V, table, c, k)
        n = int(c[-1])
        assert torch.equal(out[0][:n], want[0][:n]) and torch.equal(out[1][:n], want[1][:n])
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()


def test_bad_lengths_and_pages_are_reported_and_contained():
    lens = [(100, 3), (200, 2), (70, 4)]
    Q, K, V, table, cu, kv = _case(lens, 2, 1, 64, poison=False)
    ch = sas.SasChunk(3, 2, 1, 64, table.shape[1], K.shape[0], 9)
    good, _ = ch.attention(Q, K, V, table, cu, kv)

    def run(table=table, cu=cu, kv=kv):
        O = torch.full_like(Q, 7.0)
        ch.attention(Q, K, V, table, cu, kv, out=(O, None))
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
        return O

    for bad in (1, -5, 64 * table.shape[1] + 1):        # shorter than its new tokens, negative, past the table
        k = kv.clone()
        k[1] = bad
        O = run(kv=k)
        assert bool((O[3:5] == 7).all()) and torch.equal(O[:3], good[:3]) and torch.equal(O[5:], good[5:])
    for c in ([0, 5, 3, 9], [-1, 3, 5, 9], [0, 3, 5, 10]):   # decreasing, before and past the rows
        assert bool((run(cu=torch.tensor(c, dtype=I32, device=DEV)) == 7).all())
    for page in (-1, K.shape[0], 2 ** 31 - 1):           # reads as zero keys and values
        t = table.clone()
        t[0, 0] = page
        O = run(table=t)
        assert torch.equal(O[3:], good[3:])
        K0, V0 = torch.cat((K, torch.zeros_like(K[:1]))), torch.cat((V, torch.zeros_like(V[:1])))
        t[0, 0] = K.shape[0]
        _compare(O[:3], None, Q[:3], K0, V0, t[:1], cu[:2], kv[:1], 1 / 8)
    ch.close()


def test_timeouts_are_reported_and_the_handle_recovers():
    # a budget of one cycle makes the waits for the first work item give up: a status, no hang, and the
    # right result afterwards
    Q, K, V, table, cu, kv = _case([(3000, 1), (2000, 200)], 8, 2, 128, poison=False)
    ch = sas.SasChunk(2, 8, 2, 128, table.shape[1], K.shape[0], 201)
    want = ch.attention(Q, K, V, table, cu, kv)
    sas.sas_chunk_set_wait_limit(ch.h, 1)
    ch.attention(Q, K, V, table, cu, kv)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_TIMEOUT
    sas.sas_chunk_set_wait_limit(ch.h, 0)
    got = ch.attention(Q, K, V, table, cu, kv)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(sas.SasError):
        sas.sas_chunk_set_wait_limit(ch.h, -1)
    ch.close()


def test_refusals():
    Q, K, V, table, cu, kv = _case([(10, 2)], 2, 1, 64)
    ch = sas.SasChunk(1, 2, 1, 64, table.shape[1], K.shape[0], 2)
    with pytest.raises(sas.SasError, match="max_tokens"):
        ch.attention(Q.repeat(2, 1, 1), K, V, table, cu, kv)
    with pytest.raises(sas.SasError, match="num_seqs"):
        ch.attention(Q, K, V, table.repeat(2, 1), torch.tensor([0, 1, 2], dtype=I32, device=DEV), kv.repeat(2))
    with pytest.raises(sas.SasError, match="misaligned"):
        odd = torch.zeros(Q.numel() + 4, device=DEV, dtype=torch.bfloat16)[4:].view(Q.shape)
        ch.attention(odd, K, V, table, cu, kv)
    with pytest.raises(ValueError, match="Q must have shape"):
        ch.attention(Q[:, :1].contiguous(), K, V, table, cu, kv)
    with pytest.raises(ValueError, match="cu_new"):
        ch.attention(Q, K, V, table, cu[:1], kv)
    with pytest.raises(ValueError, match="columns"):
        ch.attention(Q, K, V, table[:, :1].contiguous(), cu, kv)
    with pytest.raises(ValueError, match="contiguous"):
        ch.attention(Q.transpose(0, 1).contiguous().transpose(0, 1), K, V, table, cu, kv)
    with pytest.raises(ValueError, match="O must"):
        ch.attention(Q, K, V, table, cu, kv, out=(Q.float(), None))
    assert sas.sas_chunk_launch_count(ch.h) == 0
    ch.attention(Q, K, V, table, cu, kv)
    assert sas.sas_chunk_launch_count(ch.h) == 2
    ch.close()
