"""The example's server when a page plan is refused: nobody gets anything, the lengths stay, and the next step that
fits goes on as if the refused one had not been asked for."""
import pytest
import torch

from examples import serving as X
from paper_2609_13141_gb300 import sas
from tests import parity as P
from tests.test_gpu_serving_example import _dense, _rel

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _server():
    s = X.Server(3, 4, 2, 64, 192, 80, topk=32)
    x = [s.projection(n) for n in (60, 33, 63)]
    s.prefill(x)
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_OK
    return s, x


def _draft(s, n=4, V=40):
    B = s.B
    probs = torch.softmax(torch.randn(B * n, V, generator=s.g, device=DEV), -1)
    drafts = torch.multinomial(probs, 1, generator=s.g).to(torch.int32).view(B, n)
    seen = []

    def target(O):
        seen.append(O.clone())
        t = torch.full((B, n + 1, V), 1.0 / V, device=DEV)
        t[:, :n] = probs.view(B, n, V)     # every draft is accepted
        return t.view(-1, V)

    y = s.projection(B * (n + 1))
    return y, s.drafted(y, drafts, probs, target), seen[0]


def test_a_drafted_step_without_pages_changes_nothing():
    s, x = _server()
    lens, table, held = s.lens.clone(), s.table.clone(), s.held.clone()
    K, V = s.K.clone(), s.V.clone()
    taken = s.taken.clone()
    s.taken = torch.full_like(taken, s.free.numel())          # no page is left
    _, (accepted, tokens), O = _draft(s)
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_ERR_OOM
    assert torch.equal(s.lens, lens) and torch.equal(s.table, table) and torch.equal(s.held, held)
    assert torch.equal(s.K, K) and torch.equal(s.V, V) and int(s.taken) == s.free.numel()
    assert accepted.tolist() == [0] * 3 and bool((tokens == -1).all())
    assert not bool(O.any())                                  # no row was computed: none holds anything
    s.taken = taken                                           # pages again: the step goes through
    y, (accepted, tokens), O = _draft(s)
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_OK
    assert accepted.tolist() == [4] * 3 and torch.equal(s.lens, lens + 5)
    for b in range(3):
        want = _dense(s, torch.cat((x[b], y[5 * b:5 * b + 5])), x[b].shape[0])[x[b].shape[0]:]
        assert _rel(P.f64(O.view(3, 5, 4, 64)[b]), want) < 2.0 ** -5   # as in the example's own test
    s.close()


def test_a_decode_step_without_pages_changes_nothing():
    s, x = _server()
    y = s.projection(3)
    O, _ = s.decode(y)                                        # 61, 34, 64 tokens
    lens, taken = s.lens.clone(), s.taken.clone()
    s.taken = torch.full_like(taken, s.free.numel())
    O, _ = s.decode(s.projection(3))                          # the third would open a page
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_ERR_OOM
    assert torch.equal(s.lens, lens) and not bool(O.any())
    s.taken = taken
    O, _ = s.decode(s.projection(3))
    assert sas.sas_chunk_get_device_status(s.step.h) == sas.SAS_OK
    assert torch.equal(s.lens, lens + 1) and bool(O.isfinite().all()) and bool(O.any())
    s.close()


def test_a_prompt_without_pages_is_refused():
    s, x = _server()
    lens = s.lens.clone()
    with pytest.raises(RuntimeError, match="pages"):
        s.prefill([s.projection(n) for n in (10, 170, 1)])    # the second passes the table in its third chunk
    # what was granted before stands; the refused chunk counts for nobody
    assert (s.lens - lens).tolist() == [10, 150, 0]
    s.close()
