"""GPU page plan (block tables and slot maps) against the oracle: every value equal."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


def _t(x, dtype=I32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def _state(seq, max_blocks, spare, seed=0):
    """Table of what is held, over shuffled pages, and the rest as the free list."""
    rng = np.random.default_rng(seed)
    held = [-(-s // 64) for s in seq]
    P = max(1, sum(held) + spare)
    perm = rng.permutation(P).astype(np.int32)[:sum(held) + spare]
    table = np.full((len(seq), max_blocks), -1, dtype=np.int32)
    k = 0
    for b, c in enumerate(held):
        table[b, :c] = perm[k:k + c]
        k += c
    return table, perm[k:], P


def _check(seq, new, T, max_blocks=64, begin=0, spare=None, seed=0):
    need = sum(-(-(s + n) // 64) - -(-s // 64) for s, n in zip(seq, new))
    table, free, P = _state(seq, max_blocks, need + begin if spare is None else spare, seed)
    ch = sas.SasChunk(len(seq), 1, 1, 64, max_blocks, P, max(T, 1))
    tab = _t(table)
    p = ch.plan(_t(seq), _t(new), _t(free), _t([begin]), tab, T)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    ch.close()
    kv, cu, pos, slots, end, want = S.plan(seq, new, free, begin, table, T)
    assert p.kv_lens.tolist() == kv and p.cu_new.tolist() == cu and p.positions.tolist() == pos
    assert p.slots.tolist() == slots and p.free_end.tolist() == [end] and np.array_equal(tab.cpu().numpy(), want)


@pytest.mark.parametrize("seq,new,T", [
    ([0], [1], 1),
    ([0], [0], 1),                                   # nothing at all
    ([63, 64, 65], [1, 1, 1], 3),                    # fills, opens and stays in a page
    ([0, 0, 0, 5], [0, 0, 64, 0], 64),               # empty requests around the only one
    ([10, 0, 128, 1], [0, 130, 0, 63], 300),         # padding past the end
    ([1] * 40, [64] * 40, 2560),
])
def test_small_plans(seq, new, T):
    _check(seq, new, T)


@pytest.mark.parametrize("B,hi,seed", [(1, 4000, 1), (513, 3, 2), (700, 150, 3), (1025, 1, 4), (8192, 2, 5), (3000, 40, 6)])
def test_many_requests(B, hi, seed):
    rng = np.random.default_rng(seed)
    seq = rng.integers(0, 200, size=B).tolist()
    new = (rng.integers(0, hi + 1, size=B) * (rng.random(B) < 0.8)).tolist()
    _check(seq, new, max(1, sum(new)) + seed, max_blocks=66, begin=seed, seed=seed)


def test_exact_fit_of_pages_and_tokens():
    _check([0, 64], [128, 64], 192, spare=3)


@pytest.mark.parametrize("what", ["pages", "tokens", "negative", "long", "begin", "begin_past", "sum"])
def test_what_does_not_fit_changes_nothing(what):
    seq, new, T, begin, spare = [10, 64, 0], [60, 1, 200], 261, 0, 6
    status = sas.SAS_ERR_INVALID_ARG
    if what == "pages":
        spare, status = 5, sas.SAS_ERR_OOM
    elif what == "tokens":
        T = 260
    elif what == "negative":
        new[1] = -1
    elif what == "long":
        new[1] = 64 * 8
    elif what == "begin":
        begin = -1
    elif what == "begin_past":
        begin = 7
    elif what == "sum":
        seq, new = [0] * 3, [512] * 3
    table, free, P = _state(seq, 8, spare)
    ch = sas.SasChunk(3, 1, 1, 64, 8, P, T)
    tab = _t(table)
    p = ch.plan(_t(seq), _t(new), _t(free), _t([begin]), tab, T)
    assert sas.sas_chunk_get_device_status(ch.h) == status
    assert p.kv_lens.tolist() == seq and p.cu_new.tolist() == [0] * 4 and p.free_end.tolist() == [begin]
    assert p.positions.tolist() == [-1] * T and p.slots.tolist() == [-1] * T
    assert np.array_equal(tab.cpu().numpy(), table)
    ch.close()


def test_lengths_whose_sum_passes_32_bits():
    # 8192 requests of 2^21 tokens: 2^34 in all, refused and not wrapped
    ch = sas.SasChunk(8192, 1, 1, 64, 32768, 10, 64)
    tab = torch.full((8192, 32768), -1, dtype=I32, device=DEV)
    p = ch.plan(_t([0] * 8192), _t([1 << 21] * 8192), _t(list(range(10))), _t([0]), tab, 64)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
    assert int(p.cu_new.abs().sum()) == 0 and bool((tab == -1).all())
    p = ch.plan(_t([2 ** 31 - 1] * 8192), _t([2 ** 31 - 1] * 8192), _t(list(range(10))), _t([0]), tab, 64)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG and int(p.cu_new.abs().sum()) == 0
    ch.close()


def test_pages_outside_the_cache_take_their_tokens_out():
    ch = sas.SasChunk(3, 1, 1, 64, 4, 10, 200)
    tab = _t([[99, -1, -1, -1], [2, -1, -1, -1], [3, -1, -1, -1]])
    p = ch.plan(_t([10, 64, 63]), _t([2, 3, 66]), _t([10, 5, -4, 6]), _t([0]), tab, 71)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG
    # request 0 continues page 99; request 1 opens page 10; request 2 fills page 3, then pages 5 and -4
    slots = p.slots.tolist()
    assert slots[:5] == [-1] * 5 and slots[5] == 3 * 64 + 63 and slots[6:70] == list(range(5 * 64, 6 * 64)) and slots[70] == -1
    assert [i for i, x in enumerate(p.positions.tolist()) if x < 0] == [0, 1, 2, 3, 4, 70]
    assert tab.tolist() == [[99, -1, -1, -1], [2, -1, -1, -1], [3, 5, -1, -1]]
    assert p.kv_lens.tolist() == [12, 67, 129] and p.free_end.tolist() == [3]
    ch.close()


def test_refusals():
    ch = sas.SasChunk(2, 1, 1, 64, 4, 10, 8)
    tab = torch.full((2, 4), -1, dtype=I32, device=DEV)
    seq, new, free, begin = _t([0, 0]), _t([1, 1]), _t([1, 2, 3]), _t([0])
    with pytest.raises(sas.SasError, match="max_tokens"):
        ch.plan(seq, new, free, begin, tab, 9)
    with pytest.raises(sas.SasError, match="num_seqs"):
        ch.plan(_t([0] * 3), _t([0] * 3), free, begin, torch.full((3, 4), -1, dtype=I32, device=DEV), 8)
    out = ch.plan_buffers(2, 8, DEV)
    with pytest.raises(sas.SasError, match="inputs"):
        ch.plan(seq, new, free, begin, tab, 8, out=out._replace(kv_lens=seq))
    with pytest.raises(sas.SasError, match="inputs"):
        ch.plan(seq, new, free, begin, tab, 8, out=out._replace(free_end=begin))
    with pytest.raises(ValueError, match="columns"):
        ch.plan(seq, new, free, begin, tab[:, :3].contiguous(), 8)
    with pytest.raises(ValueError, match="new_lens"):
        ch.plan(seq, new.long(), free, begin, tab, 8)
    with pytest.raises(ValueError, match="contiguous"):
        ch.plan(seq, new, free, begin, torch.full((4, 2), -1, dtype=I32, device=DEV).t(), 8)
    assert sas.sas_chunk_launch_count(ch.h) == 0
    ch.close()


def test_no_free_pages_needed():
    # an empty free list is fine while every token fits the pages held
    ch = sas.SasChunk(1, 1, 1, 64, 4, 10, 8)
    tab = _t([[7, -1, -1, -1]])
    p = ch.plan(_t([3]), _t([8]), torch.zeros(0, dtype=I32, device=DEV), _t([0]), tab, 8)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    assert p.slots.tolist() == [7 * 64 + 3 + i for i in range(8)]
    ch.close()


@pytest.mark.parametrize("seq,held,new", [
    ([62, 10, 130], [66, 10, 200], [3, 60, 62]),        # a held page opened by rejected drafts is used, not replaced
    ([1, 64, 0], [300, 64, 65], [5, 64, 200]),           # held far past the new tokens; exactly at a boundary
    ([70, 5], [0, 3], [10, 70]),                         # held below the length counts as the length
])
def test_held_pages_are_used_before_free_ones(seq, held, new):
    T = sum(new)
    top = [max(s, h) for s, h in zip(seq, held)]
    need = sum(max(0, -(-(s + n) // 64) - -(-h // 64)) for s, n, h in zip(seq, new, top))
    table, free, P = _state(top, 8, need)
    ch = sas.SasChunk(len(seq), 1, 1, 64, 8, P, T)
    tab = _t(table)
    p = ch.plan(_t(seq), _t(new), _t(free), _t([0]), tab, T, held_lens=_t(held))
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    kv, cu, pos, slots, end, want = S.plan(seq, new, free, 0, table, T, top)
    assert p.kv_lens.tolist() == kv and p.cu_new.tolist() == cu and p.positions.tolist() == pos
    assert p.slots.tolist() == slots and p.free_end.tolist() == [end] == [need] and np.array_equal(tab.cpu().numpy(), want)
    for bad in (-1, 64 * 8 + 1):
        p = ch.plan(_t(seq), _t(new), _t(free), _t([0]), tab, T, held_lens=_t([bad] + held[1:]))
        assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_ERR_INVALID_ARG and p.cu_new.tolist() == [0] * (len(seq) + 1)
    with pytest.raises(sas.SasError, match="inputs"):
        h = _t(held)
        ch.plan(_t(seq), _t(new), _t(free), _t([0]), tab, T, held_lens=h, out=p._replace(kv_lens=h))
    ch.close()


@pytest.mark.parametrize("off", [0, 1, 2])
def test_outputs_of_any_alignment(off):
    # capacity and addresses that four-token stores do not fit, with a canary behind each output
    seq, new, T = [60, 0, 130, 5], [7, 1, 66, 0], 77
    need = sum(-(-(s + n) // 64) - -(-s // 64) for s, n in zip(seq, new))
    table, free, P = _state(seq, 8, need)
    ch = sas.SasChunk(4, 1, 1, 64, 8, P, T)
    out = ch.plan_buffers(4, T, DEV)
    pos = torch.full((T + off + 8,), 77, dtype=I32, device=DEV)
    slots = torch.full((T + off + 8,), 77, dtype=torch.int64, device=DEV)
    out = out._replace(positions=pos[off:off + T], slots=slots[off:off + T])
    p = ch.plan(_t(seq), _t(new), _t(free), _t([0]), _t(table), T, out=out)
    assert sas.sas_chunk_get_device_status(ch.h) == sas.SAS_OK
    _, _, want_pos, want_slots, _, _ = S.plan(seq, new, free, 0, table, T)
    assert p.positions.tolist() == want_pos and p.slots.tolist() == want_slots
    assert bool((pos[:off] == 77).all()) and bool((pos[off + T:] == 77).all())
    assert bool((slots[:off] == 77).all()) and bool((slots[off + T:] == 77).all())
    ch.close()
