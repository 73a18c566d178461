"""GPU append into the 8-bit cache against the fp64 oracle.

A key is an fp32 chain of fewer than 16 roundings and two sums of d (norm, weight, rotation), off by at most e = 2^-19 of the
row's largest |w xh| before its rounding to e4m3, which is off by half a step: 2^-4 of the value, or 2^-10 where the step is
2^-9.  Values are exact until then.  A page whose maximum is within e of a power of two's border may have either scale."""
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
E4 = torch.float8_e4m3fn
REL = 2.0 ** -19


def _case(lens, Hq, Hkv, d, rot, seed=0, std=1.5, pad=0):
    """lens: (cached, new) of each request; pages shuffled, held ones with codes and scales, the others NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    need = [-(-(c + n) // 64) for c, n in lens]
    pages = sum(need) + 2
    perm = torch.randperm(pages, generator=g, device=DEV).tolist()
    K = torch.full((pages, Hkv, 64, d), 0x7F, dtype=torch.uint8, device=DEV)
    V, sk = K.clone(), torch.full((pages, Hkv), math.nan, device=DEV)
    sv = sk.clone()
    slots, pos, at = [], [], 0
    for (c, n), m in zip(lens, need):
        mine = perm[at:at + m]
        at += m
        for p in range(c, c + n):
            slots.append(mine[p // 64] * 64 + p % 64)
            pos.append(p)
        if c % 64 and n:
            p = mine[c // 64]
            for x, s in ((K, sk), (V, sv)):
                x[p] = torch.randn(Hkv, 64, d, generator=g, device=DEV).mul(60).to(E4).view(torch.uint8)
                s[p] = 2.0 ** torch.randint(-9, -4, (Hkv,), generator=g, device=DEV).float()
    T, H = len(slots), Hq + 2 * Hkv
    qkv = (torch.randn(T + pad, H, d, generator=g, device=DEV) * std).to(torch.bfloat16)
    qkv *= torch.exp2(torch.randint(-2, 3, (T + pad, 1, 1), generator=g, device=DEV).to(torch.bfloat16))
    w = [(1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2)]
    ang = torch.rand(max(pos, default=0) + 1, rot // 2, generator=g, device=DEV) * 6.28
    return dict(qkv=qkv, wq=w[0], wk=w[1], cos=ang.cos(), sin=ang.sin(),
                positions=torch.tensor(pos + [-1] * pad, dtype=I32, device=DEV),
                slots=torch.tensor(slots + [-1] * pad, dtype=torch.int64, device=DEV),
                K_cache=K.view(E4), V_cache=V.view(E4), K_scale=sk, V_scale=sv)


def _check(case, before, Q, Hq, eps, inter):
    """case: the caches after; before: clones of them before the call."""
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    slots = case["slots"].tolist()
    args = [f(case[k]) for k in ("qkv", "wq", "wk", "cos", "sin")] + [case["positions"].tolist(), slots, Hq, eps, inter]
    ref = S.append8(*args, *(f(before[k]) for k in ("K_cache", "V_cache", "K_scale", "V_scale")))
    live = [t for t, s in enumerate(slots) if s >= 0]
    got = f(Q)[live]
    assert (np.abs(got - ref[0][live]) <= 2.0 ** -8 * np.abs(ref[0][live]) + REL * np.abs(ref[0][live]).max(-1, keepdims=True)).all()
    # the largest |w xh| of each row, for the keys' error
    touched = {}
    for t in live:
        touched.setdefault(slots[t] // 64, set()).add(slots[t] % 64)
    for name, codes, scale in (("K", ref[1], ref[3]), ("V", ref[2], ref[4])):
        now, old = case[name + "_cache"].view(torch.uint8).cpu().numpy(), before[name + "_cache"].view(torch.uint8).cpu().numpy()
        value, s = f(case[name + "_cache"]), f(case[name + "_scale"])
        s_old = f(before[name + "_scale"])
        for p in range(now.shape[0]):
            if p not in touched:
                assert (now[p] == old[p]).all() and np.array_equal(s[p], s_old[p], equal_nan=True)
                continue
            rows = sorted(touched[p])
            rest = [r for r in range(64) if r not in touched[p]]
            for g in range(now.shape[1]):
                want = codes[p, g, rows]
                top = np.abs(want[np.isfinite(want)]).max(initial=0.0) * scale[p, g]
                if s[p, g] != scale[p, g]:
                    assert name == "K" and abs(math.log2(max(top, 1e-300) / 448) % 1 - 0.5) > 0.5 - 2 * REL, (name, p, g, s[p, g], scale[p, g])
                    want = want * (scale[p, g] / s[p, g])
                size = np.nanmax(np.abs(np.where(np.isfinite(want), want, 0)), axis=-1, keepdims=True)
                tol = np.maximum(np.abs(want) * (2.0 ** -4 + 2.0 ** -20), 2.0 ** -10) + (2 * REL * size if name == "K" else 0)
                assert (np.isnan(value[p, g, rows]) == ~np.isfinite(want)).all()
                ok = np.isfinite(want)
                assert (np.abs(value[p, g, rows] - want)[ok] <= np.broadcast_to(tol, want.shape)[ok]).all(), (name, p, g)
                if 0 in rows or s[p, g] == s_old[p, g]:
                    assert (now[p, g, rest] == old[p, g, rest]).all()
                else:      # rounded again, exactly so
                    again = S.round_e4m3(f(before[name + "_cache"])[p, g, rest] * (s_old[p, g] / s[p, g]))
                    assert np.array_equal(value[p, g, rest], again, equal_nan=True)


def _run(lens, Hq, Hkv, d, rot=None, inter=False, seed=0, std=1.5, pad=0, eps=1e-6, edit=None):
    case = _case(lens, Hq, Hkv, d, rot or d, seed, std, pad)
    if edit:
        edit(case)
    before = {k: v.clone() for k, v in case.items()}
    pages = case["K_scale"].shape[0]
    ch = sas.SasChunk(len(lens), Hq, Hkv, d, 64, pages, case["qkv"].shape[0])
    Q = ch.append8(**case, eps=eps, interleaved=inter)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    _check(case, before, Q, Hq, eps, inter)
    again = {k: v.clone() for k, v in before.items()}
    Q2 = ch.append8(**again, eps=eps, interleaved=inter)
    n = before["qkv"].shape[0] - pad
    assert torch.equal(Q[:n], Q2[:n]) and all(torch.equal(again[k].view(torch.uint8), case[k].view(torch.uint8)) for k in ("K_cache", "V_cache"))
    ch.close()
    return case, Q


# runs of one token, a few, eight and nine, a page and more; requests that begin in a page and at its start
LENS = [(0, 1), (5, 1), (64, 1), (63, 2), (10, 8), (10, 9), (0, 64), (64, 65), (60, 70), (0, 0), (3, 0), (130, 200), (7, 57), (7, 58)]


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 128), (3, 3, 64), (8, 1, 64), (1, 1, 128)])
@pytest.mark.parametrize("inter", [False, True])
def test_lengths(Hq, Hkv, d, inter):
    _run(LENS, Hq, Hkv, d, inter=inter, seed=Hq + d, pad=3)


@pytest.mark.parametrize("d,rot", [(128, 64), (128, 16), (64, 32), (64, 48)])
@pytest.mark.parametrize("inter", [False, True])
def test_part_of_a_head_turned(d, rot, inter):
    _run([(0, 70), (33, 1), (64, 12)], 4, 2, d, rot, inter)


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 64, 65])
def test_one_request(n):
    _run([(0, n)], 2, 1, 64, seed=n)
    _run([(37, n)], 2, 1, 128, seed=n)


def test_many_single_tokens():
    rng = np.random.default_rng(3)
    _run([(int(c), 1) for c in rng.integers(0, 300, 150)], 8, 4, 64, seed=9)


def test_scale_grows_keeps_and_starts_over():
    """One page written a token at a time: values grow, shrink, and the page starts over."""
    d = 64
    ch = sas.SasChunk(1, 1, 1, d, 4, 1, 1)
    one = torch.ones(d, device=DEV, dtype=torch.bfloat16)
    K = torch.zeros(1, 1, 64, d, device=DEV).to(E4)
    V, sk, sv = K.clone(), torch.full((1, 1), 7.0, device=DEV), torch.full((1, 1), math.nan, device=DEV)
    cos, sin = torch.ones(64, d // 2, device=DEV), torch.zeros(64, d // 2, device=DEV)
    sizes = [1.0, 448.0, 1.0, 500.0, 3.0, 2.0 ** 20, 2.0 ** 20]
    scales = [2.0 ** -8, 1.0, 1.0, 2.0, 2.0, 2.0 ** 12, 2.0 ** 12]
    for i, (x, s) in enumerate(zip(sizes, scales)):
        qkv = torch.full((1, 3, d), x, device=DEV, dtype=torch.bfloat16)
        ch.append8(qkv, one, one, cos, sin, torch.tensor([i], dtype=I32, device=DEV), torch.tensor([i], device=DEV), K, V, sk, sv)
        assert float(sv[0, 0]) == s and float(sk[0, 0]) == 2.0 ** -8          # normed keys stay at 1
        assert float(V[0, 0, i, 0].float()) == float(torch.tensor(float(qkv[0, 2, 0]) / s).to(E4).float())
    assert float(V[0, 0, 0, 0].float()) == 0.0 and float(V[0, 0, 1, 0].float()) == float(torch.tensor(448 / 2.0 ** 12).to(E4).float())
    qkv = torch.full((1, 3, d), 1.0, device=DEV, dtype=torch.bfloat16)
    ch.append8(qkv, one, one, cos, sin, torch.tensor([64 - 1], dtype=I32, device=DEV), torch.tensor([0], device=DEV), K, V, sk, sv)
    assert float(sv[0, 0]) == 2.0 ** -8 and float(V[0, 0, 0, 0].float()) == 256.0
    ch.close()


def test_infinities_nan_zeros_and_the_largest_numbers():
    def edit(case):
        v = case["qkv"][:, -1]           # the last value head
        v[0, 3], v[1, 4], v[2, 5] = math.inf, -math.inf, math.nan
        v[66] = 3.3895e38
        v[67] = -1e-38
        case["qkv"][130:, -1] = 0.0      # from 192 on a page of nothing but zeros
    case, _ = _run([(0, 200), (5, 1)], 4, 2, 64, edit=edit)
    assert float(case["V_scale"][int(case["slots"][195]) // 64, 1]) == 2.0 ** -64
    assert float(case["V_scale"][int(case["slots"][66]) // 64, 1]) == 2.0 ** 120


def test_strided_tokens_and_pages_past_two_to_the_31_bytes():
    case = _case([(10, 3), (64, 70)], 8, 8, 128, 128)
    T = case["qkv"].shape[0]
    wide = torch.zeros(T, 25 * 128, device=DEV, dtype=torch.bfloat16)
    wide[:, :24 * 128] = case["qkv"].view(T, -1)
    pages, far = case["K_scale"].shape[0], 41000
    a, b = sas.SasChunk(2, 8, 8, 128, 4, pages, T), sas.SasChunk(2, 8, 8, 128, 4, far, T)
    big = {k: torch.empty((far,) + case[k].shape[1:], dtype=case[k].dtype, device=DEV) for k in ("K_cache", "V_cache", "K_scale", "V_scale")}
    move = far - pages
    for k in big:
        big[k][move:] = case[k]
    Q = a.append8(**case)
    Q2 = b.append8(wide[:, :24 * 128].view(T, 24, 128), case["wq"], case["wk"], case["cos"], case["sin"], case["positions"],
                   case["slots"] + 64 * move, **big)
    assert torch.equal(Q, Q2)
    for k in big:
        x, y = (t.contiguous().view(torch.uint8) for t in (big[k][move:], case[k]))
        assert torch.equal(x, y)
    assert sas.sas_chunk_get_device_status(b.h) == sas.SAS_OK


def test_bad_slots_and_positions_are_reported_and_contained():
    case = _case([(0, 20), (70, 4)], 2, 1, 64, 64)
    pages, T = case["K_scale"].shape[0], 24
    ch = sas.SasChunk(2, 2, 1, 64, 4, pages, T)
    good = {k: v.clone() for k, v in case.items()}
    ch.append8(**good)
    for name, value in (("slots", 64 * pages), ("slots", -2), ("positions", case["cos"].shape[0]), ("positions", -1)):
        bad = {k: v.clone() for k, v in case.items()}
        bad[name][23] = value
        Q = torch.full((T, 2, 64), 7.0, device=DEV, dtype=torch.bfloat16)
        ch.append8(**bad, out=Q)
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
        assert (Q[23] == 7).all() and (Q[22] != 7).any()
        p, r = int(case["slots"][23]) // 64, int(case["slots"][23]) % 64
        for k in ("K_cache", "V_cache"):
            x, y, z = (t[k].view(torch.uint8) for t in (bad, good, case))
            keep = torch.ones(64, dtype=torch.bool, device=DEV)
            keep[r] = False
            others = torch.arange(pages, device=DEV) != p
            assert torch.equal(x[others], y[others])
            if float(bad[k[0] + "_scale"][p, 0]) == float(case[k[0] + "_scale"][p, 0]):
                assert torch.equal(x[p, :, r], z[p, :, r])
    # every token of a page bad: nothing of it changes
    bad = {k: v.clone() for k, v in case.items()}
    bad["positions"][20:] = 1 << 30
    ch.append8(**bad)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
    p = int(case["slots"][23]) // 64
    assert torch.equal(bad["V_cache"].view(torch.uint8)[p], case["V_cache"].view(torch.uint8)[p]) and torch.equal(bad["V_scale"][p], case["V_scale"][p])


def test_refusals():
    case = _case([(0, 4)], 2, 1, 64, 64)
    ch = sas.SasChunk(1, 2, 1, 64, 4, case["K_scale"].shape[0], 4)
    for k, bad in (("K_cache", case["K_cache"].view(torch.uint8)), ("V_cache", case["V_cache"].to(torch.bfloat16)), ("K_scale", case["K_scale"].double()),
                   ("V_scale", case["V_scale"][:1]), ("K_scale", case["K_scale"].t().contiguous().t()[:, :0]), ("K_cache", case["K_cache"][:-1]),
                   ("slots", case["slots"].int()), ("qkv", case["qkv"].float()), ("K_scale", case["K_scale"].cpu())):
        with pytest.raises(ValueError):
            ch.append8(**{**case, k: bad})
    with pytest.raises(sas.SasError, match="max_tokens"):
        ch.append8(**{**case, "qkv": case["qkv"].repeat(2, 1, 1), "positions": case["positions"].repeat(2), "slots": case["slots"].repeat(2)})
    assert sas.sas_chunk_launch_count(ch.h) == 0
    ch.append8(**case)
    assert sas.sas_chunk_launch_count(ch.h) == 1
    ch.close()


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 8, 64), (16, 8, 128)])
def test_batches_of_wide_windows(Hq, Hkv, d):
    """So many tokens that a block looks at more than eight at a time: the bits of the same requests a few at a time."""
    rng = np.random.default_rng(d)
    lens = [(int(rng.integers(0, 200)), n) for n in [1] * 900 + [5, 9, 64, 65, 130] * 4 + [1000, 777, 2000, 1500] + [1] * 70]
    case = _case(lens, Hq, Hkv, d, d)
    T, pages = case["qkv"].shape[0], case["K_scale"].shape[0]
    assert T * Hkv > 40 * 8 * torch.cuda.get_device_properties(0).multi_processor_count
    few = {k: v.clone() for k, v in case.items()}
    ch = sas.SasChunk(len(lens), Hq, Hkv, d, 64, pages, T)
    Q = ch.append8(**case)
    at, parts = 0, []
    while at < T:          # whole requests
        n, t = at, 0
        for _, new in lens:
            if t >= at and t + new - at <= max(400, new):
                n = t + new
            t += new
        part = {k: v[at:n] if k in ("qkv", "positions", "slots") else v for k, v in few.items()}
        parts.append(ch.append8(**part))
        at = n
    assert len(parts) > 5 and torch.equal(torch.cat(parts), Q)
    assert all(torch.equal(few[k].view(torch.uint8), case[k].view(torch.uint8)) for k in ("K_cache", "V_cache"))
    live = (case["slots"] // 64).unique()
    assert all(torch.equal(few[k][live], case[k][live]) for k in ("K_scale", "V_scale"))
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK


def test_captured_and_on_another_stream():
    case = _case([(0, 70), (5, 1), (64, 9), (10, 1)], 4, 2, 128, 128)
    start = {k: v.clone() for k, v in case.items()}
    ch = sas.SasChunk(4, 4, 2, 128, 64, case["K_scale"].shape[0], 81)
    want = {k: v.clone() for k, v in case.items()}
    Q = ch.append8(**want)
    out, side = torch.empty_like(Q), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ch.append8(**case, out=out)
    for _ in range(2):
        for k in ("K_cache", "V_cache", "K_scale", "V_scale"):
            case[k].copy_(start[k])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, Q)
        for k in ("K_cache", "V_cache", "K_scale", "V_scale"):
            assert torch.equal(case[k].contiguous().view(torch.uint8), want[k].contiguous().view(torch.uint8)), k
