"""GPU attention over an 8-bit paged cache against a plain one in 64 bits.

Bounds, element by element.  A logit is an fp32 sum of d products, off by at most delta = 2^-17 scale sum |q||k|, which moves
O by 2 delta A, A the output on |V|; the weights are rounded to fp16, 2^-11 of p |v|, or 2^-25 where that is less than 2^-14,
of weights that are scaled by at least 1 / R, R the spread of the value scales (capped at 2^6 by the kernel); fp32 sums add
2^-16 A, and the output is rounded to bf16, 2^-8 of it.  LSE moves by delta and 2^-15."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32
E4 = torch.float8_e4m3fn


def _case(lens, Hq, Hkv, d, seed=0, spare=2, std=1.0, spread=2, poison=True):
    """lens: (cached, new).  Scales within 2^-spread .. 2^spread of their heads'; what no token sees is NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    total = [c + n for c, n in lens]
    need = [-(-t // 64) for t in total]
    pages, width = sum(need) + spare, max(max(need), 1) + 1
    perm = torch.randperm(pages, generator=g, device=DEV).to(I32)
    table = torch.full((len(lens), width), -1, dtype=I32, device=DEV)
    out = []
    for _ in range(2):
        s = 2.0 ** (torch.randint(-spread, spread + 1, (pages, Hkv), generator=g, device=DEV).float() - 7)
        x = (torch.randn(pages, Hkv, 64, d, generator=g, device=DEV) / s[..., None, None]).clamp(-448, 448).to(E4)
        out += [x, s]
    K, sk, V, sv = out
    k = 0
    for b, c in enumerate(need):
        table[b, :c] = perm[k:k + c]
        k += c
        if poison and total[b] % 64:
            for x in (K, V):
                x.view(torch.uint8)[int(perm[k - 1]), :, total[b] % 64:] = 0x7F
    if poison:
        for p in perm[k:].tolist():
            K.view(torch.uint8)[p], V.view(torch.uint8)[p], sk[p], sv[p] = 0x7F, 0xFF, math.nan, math.nan
    cu = torch.tensor([0] + np.cumsum([n for _, n in lens]).tolist(), dtype=I32, device=DEV)
    Q = (torch.randn(int(cu[-1]), Hq, d, generator=g, device=DEV) * std).to(torch.bfloat16)
    return Q, K, V, sk, sv, table, cu, torch.tensor(total, dtype=I32, device=DEV)


def _plain(Q, K, V, sk, sv, table, cu, kv, scale):
    """O, LSE, A, S, U: S the largest scale sum |q||k| of a row, U = sum |v| / sum exp(z - max)."""
    T, Hq, d = Q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    f64 = dict(dtype=torch.float64, device=DEV)
    O, A, U = (torch.full((T, Hq, d), math.nan, **f64) for _ in range(3))
    LSE, size = torch.full((T, Hq), math.nan, **f64), torch.full((T, Hq), math.nan, **f64)
    for b, L in enumerate(kv.tolist()):
        t0, t1 = int(cu[b]), int(cu[b + 1])
        if t0 == t1:
            continue
        pages = table[b, :-(-L // 64)].long()
        for g in range(Hkv):
            k, v = ((x.view(torch.uint8)[pages, g].view(E4).double() * s[pages, g].double()[:, None, None]).reshape(-1, d)[:L] for x, s in ((K, sk), (V, sv)))
            q = Q[t0:t1, g * G:(g + 1) * G].double()
            late = torch.arange(L, device=DEV) > (L - (t1 - t0) + torch.arange(t1 - t0, device=DEV))[:, None]
            z = (torch.einsum("tgd,ld->tgl", q, k) * scale).masked_fill(late[:, None], -math.inf)
            at = slice(t0, t1), slice(g * G, (g + 1) * G)
            top = z.amax(-1, keepdim=True)
            e = (z - top).exp()
            n = e.sum(-1, keepdim=True)
            O[at], A[at] = e @ v / n, e @ v.abs() / n
            U[at] = (~late).double()[:, None] @ v.abs() / n
            LSE[at] = (top + n.log())[..., 0]
            size[at] = torch.einsum("tgd,ld->tgl", q.abs(), k.abs()).masked_fill(late[:, None], 0).amax(-1) * scale
    return O, LSE, A, size, U


def _compare(O, LSE, case, scale, R=16.0):
    ref, lse, A, size, U = _plain(*case, scale)
    live = ~lse.isnan()
    delta = 2.0 ** -17 * size
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2.0 ** -16 + 2 * delta[..., None]) * A + 2.0 ** -25 * R * U
    err = (O.double() - ref).abs()
    assert O[live].isfinite().all()
    assert (err[live] <= tol[live]).all(), f"O: worst {float((err - tol)[live].max()):.3g} over the bound"
    if LSE is not None:
        e = (LSE.double() - lse).abs()
        assert (e[live] <= (delta + 2.0 ** -15)[live]).all(), f"LSE off by {float(e[live].max()):.3g}"


def _chunk(case, scale=0.0, T=None):
    Q, K, _, _, _, table, _, kv = case
    return sas.SasChunk(kv.shape[0], Q.shape[1], K.shape[1], Q.shape[2], table.shape[1], K.shape[0], T or max(Q.shape[0], 1), scale)


def _run(lens, Hq, Hkv, d, seed=0, scale=0.0, std=1.0, **kw):
    case = _case(lens, Hq, Hkv, d, seed, std=std, **kw)
    ch = _chunk(case, scale)
    O, LSE = ch.attention8(*case)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    O2, LSE2 = ch.attention8(*case)
    assert torch.equal(O, O2) and torch.equal(LSE, LSE2)   # equal inputs, equal bits, split or not
    ch.close()
    _compare(O, LSE, case, scale or 1 / math.sqrt(d))


def test_plain_form_is_the_oracles():
    case = _case([(70, 3), (0, 2)], 4, 2, 64, poison=False)
    Q, K, V, sk, sv, table, cu, kv = case
    ref = _plain(*case, 0.125)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    deq = [f(x) * f(s)[..., None, None] for x, s in ((K, sk), (V, sv))]
    O, LSE, A, _ = S.chunk_attention(f(Q), *deq, table.cpu().numpy(), cu.tolist(), kv.tolist(), 0.125)
    for a, b in ((ref[0], O), (ref[1], LSE), (ref[2], A)):
        assert np.abs(f(a) - b).max() < 1e-12


GD = [(1, 64), (2, 128), (4, 128), (8, 64), (1, 128), (4, 64), (8, 128), (2, 64)]


@pytest.mark.parametrize("G,d", GD)
def test_single_tokens(G, d):
    # one row of the group a token: the first token, page boundaries on either side, long and short ones together
    _run([(c, 1) for c in (0, 1, 62, 63, 64, 65, 127, 128, 500, 1500, 3)] + [(100, 0), (0, 0)], 2 * G, 2, d, seed=G + d)
    _run([(2500, 1)], G, 1, d, seed=G)


@pytest.mark.parametrize("G,d", GD)
@pytest.mark.parametrize("n", [2, 3, 5, 8])
def test_a_few_tokens(G, d, n):
    _run([(0, n), (63, n), (61, n), (700, n), (64 - n, n), (2000, n)], G, 1, d, seed=n)


@pytest.mark.parametrize("G,d", GD)
def test_lengths_that_meet_every_edge(G, d):
    lens = [(0, 1), (0, 63), (0, 64), (0, 65), (63, 1), (64, 1), (65, 2), (127, 129), (200, 0), (0, 0), (31, 130), (300, 17)]
    _run(lens, 2 * G, 2, d, seed=G + d)


@pytest.mark.parametrize("G,Hkv,d,lens", [
    (8, 1, 64, [(5000, 3), (10, 1)]),
    (1, 3, 128, [(2000, 40)]),
    (2, 1, 64, [(700, 128), (1, 1), (64, 64)]),
    (4, 8, 128, [(1500, 5)] * 3),
    (1, 1, 64, [(0, 700)]),
    (4, 2, 128, [(64 * k + 7, 1 + 5 * k) for k in range(20)]),
    (8, 1, 128, [(19000, 1)]),                      # one unit of many splits
    (1, 1, 64, [(6000, 128)]),
    (4, 1, 128, [(4500, 33)]),
    (1, 1, 128, [(600, 1)]),
    (2, 2, 64, [(9000, 7), (300, 1)]),
    (8, 4, 128, [(300, 300), (5, 700)]),
])
def test_splits_and_mixed_batches(G, Hkv, d, lens):
    _run(lens, G * Hkv, Hkv, d, seed=len(lens))


@pytest.mark.parametrize("G,Hkv,lens", [(1, 4, [(9000, 1300)]), (2, 4, [(9000, 2195)]), (4, 8, [(9000, 1500)]), (8, 4, [(5000, 715)]),
                                        (4, 4, [(3000, 411), (5000, 400), (700, 1), (4000, 285)])])
def test_last_tiles_of_half_a_pair(G, Hkv, lens):
    # requests whose last unit fills one of a block's two tiles at most, taken ahead of a split that has both;
    # what another batch left in the block's memory shows nowhere
    case, other = (_case(lens, G * Hkv, Hkv, 128, seed=k) for k in (5, 6))
    ch = _chunk(case)
    first = None
    for _ in range(3):
        ch.attention8(*other)
        O, LSE = ch.attention8(*case)
        first = first or (O, LSE)
        assert torch.equal(O, first[0]) and torch.equal(LSE, first[1])
    _compare(O, LSE, case, 1 / math.sqrt(128))
    assert sas.sas_chunk_get_device_status(ch.h) == 0


def test_many_sequences():
    rng = np.random.default_rng(7)
    _run([(int(c), int(n)) for c, n in zip(rng.integers(0, 90, 1500), rng.integers(0, 3, 1500))], 2, 1, 64, seed=1)


@pytest.mark.parametrize("n", [1, 4, 7])
def test_long_contexts_of_many_requests(n):
    """Memory at its limit: every block walks several units of many pages, whose loads end out of order."""
    rng = np.random.default_rng(n)
    case = _case([(int(c), n) for c in np.exp(rng.uniform(np.log(100), np.log(9000), 64))], 32, 8, 128, seed=n)
    ch = _chunk(case)
    for _ in range(20):
        O, LSE = ch.attention8(*case)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    _compare(O, LSE, case, 1 / math.sqrt(128))


def test_many_heads():
    _run([(100, 1), (700, 2)], 96, 12, 64, seed=1)
    _run([(100, 1), (700, 2)], 40, 40, 128, seed=2)


@pytest.mark.parametrize("lens", [[(500, 1), (90, 1)], [(500, 5)], [(500, 30), (90, 1)], [(100, 300)]])
def test_scale_and_peaked_rows(lens):
    _run(lens, 4, 2, 128, seed=3, scale=0.9, std=4.0)      # logits of +-100: the maximum moves far and often
    _run(lens, 4, 2, 64, seed=3, scale=0.9, std=4.0)


@pytest.mark.parametrize("lens", [[(700, 1)], [(700, 6)], [(500, 200)]])
@pytest.mark.parametrize("d", [64, 128])
def test_value_scales_far_apart(lens, d):
    """Pages of 2^-50 .. 2^50: the output is that of the largest ones, and a column that is zero there is that of the small
    ones, to its own precision."""
    case = _case(lens, 4, 1, d, seed=5, poison=False)
    Q, K, V, sk, sv, table, cu, kv = case
    pages = table[0][table[0] >= 0].long()
    for i, p in enumerate(pages.tolist()):
        big = i % 3 == 1
        sv[p] = 2.0 ** (50 if big else -50)
        if big:
            V.view(torch.uint8)[p, :, :, 5] = 0
    ch = _chunk(case)
    O, LSE = ch.attention8(*case)
    ref, lse, A, size, U = _plain(*case, 1 / math.sqrt(d))
    few = torch.isfinite(ref)
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2.0 ** -16 + 2.0 ** -16 * size[..., None]) * A + 2.0 ** -25 * 64 * U
    assert ((O.double() - ref).abs()[few] <= tol[few]).all()


@pytest.mark.parametrize("lens", [[(300, 1)], [(300, 5)], [(200, 150)]])
def test_queries_of_any_size(lens):
    """Rows of 2^-100 and 2^60, and numbers of very different size in one row, keys to match."""
    case = _case(lens, 8, 2, 128, seed=6, poison=False)
    Q, K, V, sk, sv, table, cu, kv = case
    Q[:, 0] *= 2.0 ** -100
    Q[:, 4] *= 2.0 ** 60
    sk[:, 1] *= 2.0 ** -60
    Q[:, 1, ::2] *= 2.0 ** -15
    Q[:, 2, 1:] *= 2.0 ** -28
    Q[:, 3] = 0
    ch = _chunk(case)
    O, LSE = ch.attention8(*case)
    _compare(O, LSE, case, 1 / math.sqrt(128))
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


def test_rows_past_the_end_and_lse_none_are_left_alone():
    for lens in ([(100, 5), (3, 2)], [(100, 1), (3, 1)], [(100, 90), (3, 2)]):
        Q, *rest = case = _case(lens, 4, 2, 64)
        n = Q.shape[0]
        ch = _chunk(case, T=200)
        wide = torch.full((n + 9, 4, 64), float("nan"), device=DEV, dtype=torch.bfloat16)
        wide[:n] = Q
        O, LSE = torch.full_like(wide, 7.0), torch.full((n + 9, 4), 7.0, device=DEV)
        ch.attention8(wide, *rest, out=(O, LSE))
        assert bool((O[n:] == 7).all()) and bool((LSE[n:] == 7).all())
        O2 = torch.full_like(wide, 7.0)
        ch.attention8(wide, *rest, out=(O2, None))
        assert torch.equal(O, O2)
        _compare(O[:n], LSE[:n], case, 1 / 8)
        ch.close()


SHAPES = [(4, 2, 128, [(3000, 1), (500, 3)]), (8, 2, 64, [(5000, 3), (700, 1)]), (8, 1, 128, [(9000, 1)]), (1, 2, 64, [(3000, 128), (90, 5)]),
          (1, 1, 128, [(1200, 1)])]


@pytest.mark.parametrize("G,Hkv,d,lens", SHAPES)
@pytest.mark.parametrize("tail", [True, False])
def test_live_nan_keys_reach_every_row_that_sees_them(G, Hkv, d, lens, tail):
    case = _case(lens, G * Hkv, Hkv, d, seed=G + d)
    Q, K, V, sk, sv, table, cu, kv = case
    n, L = lens[0][1], int(kv[0])
    ch = _chunk(case)
    R, M = ch.attention8(*case)
    for page in range(0, -(-(L - n) // 64), 7):
        bad = K.clone()
        lo, hi = (64 * page, L) if tail else (0, min(64 * (page + 1), L - n))
        for p in range(lo // 64, -(-hi // 64)):
            bad.view(torch.uint8)[int(table[0, p]), 0, max(lo - 64 * p, 0):min(hi - 64 * p, 64)] = 0x7F
        O, LSE = ch.attention8(Q, bad, *case[2:])
        assert bool(O[:n, :G].isnan().all()) and bool(LSE[:n, :G].isnan().all()), f"page {page}"
        O[:n, :G], LSE[:n, :G] = R[:n, :G], M[:n, :G]
        assert torch.equal(O, R) and torch.equal(LSE, M)      # everything else: as without them


def test_infinite_and_nan_queries_stay_in_their_rows():
    case = _case([(500, 5), (64, 2)], 4, 2, 64)
    ch = _chunk(case)
    R, M = ch.attention8(*case)
    Q = case[0].clone()
    Q[1, 2, 7], Q[6, 0, 3] = math.nan, math.inf
    O, LSE = ch.attention8(Q, *case[1:])
    assert O[1, 2].isnan().all() and LSE[1, 2].isnan() and not O[6, 0].isfinite().all()
    for t, h in ((1, 2), (6, 0)):
        O[t, h], LSE[t, h] = R[t, h], M[t, h]
    assert torch.equal(O, R) and torch.equal(LSE, M)


def test_pages_past_two_to_the_32_bytes():
    pages, Hq, Hkv, d = 66000, 8, 8, 128
    for lens in ([(130, 3)], [(130, 1)], [(100, 60)]):
        case = _case(lens, Hq, Hkv, d, poison=False)
        Q, K, V, sk, sv, table, cu, kv = case
        big = torch.empty(2, pages, Hkv, 64, d, device=DEV, dtype=torch.uint8).view(E4)
        bs = torch.ones(2, pages, Hkv, device=DEV)
        far = torch.tensor([[pages - 1, 4, pages - 9, -1]], dtype=I32, device=DEV)
        for i in range(3):
            p, q = int(far[0, i]), int(table[0, i])
            for j, (x, s) in enumerate(((K, sk), (V, sv))):
                big[j].view(torch.uint8)[p], bs[j, p] = x.view(torch.uint8)[q], s[q]
        b = sas.SasChunk(1, Hq, Hkv, d, 4, pages, 60)
        x, y = _chunk(case).attention8(*case), b.attention8(Q, big[0], big[1], bs[0], bs[1], far, cu, kv)
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


@pytest.mark.parametrize("lens", [[(500, 9), (64, 1), (0, 40)], [(500, 1), (64, 1), (3, 1)]])
def test_replayed_graph_follows_the_lengths_on_another_stream(lens):
    case = _case(lens, 4, 1, 64, poison=False)
    Q, *rest, cu, kv = case
    ch = _chunk(case)
    out = (torch.empty_like(Q), torch.empty(Q.shape[:2], device=DEV))
    cu2, kv2 = torch.zeros_like(cu), torch.zeros_like(kv)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ch.attention8(Q, *rest, cu2, kv2, out=out, stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ch.attention8(Q, *rest, cu2, kv2, out=out, stream=side)
    for c, k in ((cu, kv), (torch.tensor([0, 1, 2, 3], dtype=I32, device=DEV), torch.tensor([501, 3, 4], dtype=I32, device=DEV))):
        cu2.copy_(c)
        kv2.copy_(k)
        g.replay()
        torch.cuda.synchronize()
        want = ch.attention8(Q, *rest, c, k)
        n = int(c[-1])
        assert torch.equal(out[0][:n], want[0][:n]) and torch.equal(out[1][:n], want[1][:n])
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


@pytest.mark.parametrize("lens", [[(100, 3), (200, 2), (70, 4)], [(100, 90), (200, 20), (70, 40)]])
def test_bad_lengths_and_pages_are_reported_and_contained(lens):
    case = _case(lens, 2, 1, 64, poison=False)
    Q, K, V, sk, sv, table, cu, kv = case
    ch = _chunk(case)
    good, _ = ch.attention8(*case)
    a, b, T = lens[0][1], lens[0][1] + lens[1][1], Q.shape[0]

    def run(table=table, cu=cu, kv=kv):
        O = torch.full_like(Q, 7.0)
        ch.attention8(Q, K, V, sk, sv, table, cu, kv, out=(O, None))
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
        return O

    for bad in (1, -5, 64 * table.shape[1] + 1):        # shorter than its new tokens, negative, past the table
        k = kv.clone()
        k[1] = bad
        O = run(kv=k)
        assert bool((O[a:b] == 7).all())
        _compare(torch.cat([O[:a], O[b:]]), None, (torch.cat([Q[:a], Q[b:]]), K, V, sk, sv, table[[0, 2]],
                                                   torch.tensor([0, a, a + T - b], dtype=I32, device=DEV), kv[[0, 2]]), 1 / 8)
    for c in ([0, b, a, T], [-1, a, b, T], [0, a, b, T + 1]):   # decreasing, before and past the rows
        assert bool((run(cu=torch.tensor(c, dtype=I32, device=DEV)) == 7).all())
    for page in (-1, K.shape[0], 2 ** 31 - 1):           # reads as zero keys and values
        t = table.clone()
        t[0, 0] = page
        O = run(table=t)
        assert torch.equal(O[a:], good[a:])
        zero = torch.zeros_like(K.view(torch.uint8)[:1])
        K0, V0 = (torch.cat((x.view(torch.uint8), zero)).view(E4) for x in (K, V))
        t[0, 0] = K.shape[0]
        one = torch.ones_like(sk[:1])
        _compare(O[:a], None, (Q[:a], K0, V0, torch.cat((sk, one)), torch.cat((sv, one)), t[:1], cu[:2], kv[:1]), 1 / 8)
    ch.close()


@pytest.mark.parametrize("lens", [[(3000, 1), (2000, 2)], [(3000, 1), (2000, 200)]])
def test_timeouts_are_reported_and_the_handle_recovers(lens):
    case = _case(lens, 8, 2, 128, poison=False)
    ch = _chunk(case)
    want = ch.attention8(*case)
    sas.sas_chunk_set_wait_limit(ch.h, 1)
    ch.attention8(*case)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_TIMEOUT
    sas.sas_chunk_set_wait_limit(ch.h, 0)
    got = ch.attention8(*case)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ch.close()


def test_steps_of_a_server():
    """plan, append8, attention8 and logprobs over steps of prompt chunks, drafts and single tokens, captured once a
    shape: the cache that grows step by step holds every token's key and value to e4m3's step (twice where its page's scale
    grew), and each step's attention is that over the cache as it stands."""
    g = torch.Generator(device=DEV).manual_seed(11)
    B, Hq, Hkv, d, P, W = 3, 8, 2, 64, 40, 8
    ch = sas.SasChunk(B, Hq, Hkv, d, W, P, 128)
    K, V = (torch.zeros(P, Hkv, 64, d, device=DEV).to(E4) for _ in range(2))
    sk, sv = torch.full((P, Hkv), math.nan, device=DEV), torch.full((P, Hkv), math.nan, device=DEV)
    table = torch.full((B, W), -1, dtype=I32, device=DEV)
    free, begin = torch.randperm(P, generator=g, device=DEV).to(I32), torch.zeros(1, dtype=I32, device=DEV)
    w = torch.ones(d, device=DEV, dtype=torch.bfloat16)
    ang = torch.rand(512, d // 2, generator=g, device=DEV)
    cos, sin = ang.cos(), ang.sin()
    lens, kept = torch.zeros(B, dtype=I32, device=DEV), [[] for _ in range(B)]
    head = torch.randn(Hq * d, 1000, generator=g, device=DEV) / 16
    for new in ([70, 10, 0], [1, 1, 90], [5, 2, 5], [1, 1, 1], [1, 1, 1], [40, 1, 3]):
        T = sum(new)
        n = torch.tensor(new, dtype=I32, device=DEV)
        plan = ch.plan(lens, n, free, begin, table, T)
        qkv = torch.randn(T, Hq + 2 * Hkv, d, generator=g, device=DEV).to(torch.bfloat16)
        Q = ch.append8(qkv, w, w, cos, sin, plan.positions, plan.slots, K, V, sk, sv)
        O, LSE = ch.attention8(Q, K, V, sk, sv, table, plan.cu_new, plan.kv_lens)
        _compare(O, LSE, (Q, K, V, sk, sv, table, plan.cu_new, plan.kv_lens), 1 / 8)
        logits = O.reshape(T, -1).float() @ head
        r = ch.logprobs(logits, logits.argmax(-1).to(I32), 3)
        assert torch.equal(r.top_index[:, 0].long(), logits.argmax(-1))
        assert (r.logprob - torch.log_softmax(logits.double(), -1).amax(-1)).abs().max() < 1e-4
        for b in range(B):
            kept[b].append(qkv[int(plan.cu_new[b]):int(plan.cu_new[b + 1]), Hq + Hkv:].float())
        lens, begin = plan.kv_lens.clone(), plan.free_end.clone()
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    for b in range(B):
        want = torch.cat(kept[b])
        pages = table[b][table[b] >= 0].long()
        got = (V.view(torch.uint8)[pages].view(E4).float() * sv[pages][..., None, None]).transpose(1, 2).reshape(-1, Hkv, d)[:want.shape[0]]
        floor = sv[pages].amax() * 2.0 ** -9
        assert ((got - want).abs() <= 2 * (want.abs() * 2.0 ** -4) * (1 + 2.0 ** -4) + 2 * floor).all()


def test_refusals():
    case = _case([(10, 2)], 2, 1, 64)
    Q, K, V, sk, sv, table, cu, kv = case
    ch = _chunk(case)
    with pytest.raises(sas.SasError, match="max_tokens"):
        ch.attention8(Q.repeat(2, 1, 1), *case[1:])
    with pytest.raises(sas.SasError, match="num_seqs"):
        ch.attention8(Q, K, V, sk, sv, table.repeat(2, 1), torch.tensor([0, 1, 2], dtype=I32, device=DEV), kv.repeat(2))
    for i, bad in ((0, Q[:, :1].contiguous()), (0, Q.float()), (1, K.view(torch.uint8)), (2, V.to(torch.bfloat16)), (3, sk[:1]), (4, sv.double()),
                   (4, sv.cpu()), (5, table[:, :1].contiguous()), (6, cu[:1]), (7, kv.long())):
        with pytest.raises(ValueError):
            ch.attention8(*case[:i], bad, *case[i + 1:])
    with pytest.raises(ValueError, match="O must"):
        ch.attention8(*case, out=(Q.float(), None))
    assert sas.sas_chunk_launch_count(ch.h) == 0
    ch.attention8(*case)
    assert sas.sas_chunk_launch_count(ch.h) == 2
    ch.close()
