"""Tensors of other sizes than their handle's are refused by the functions, not only by the classes."""
import pytest
import torch

from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32, BF = torch.int32, torch.bfloat16


def _bf(*shape):
    return torch.zeros(*shape, device=DEV, dtype=BF)


def _ints(*shape):
    return torch.zeros(*shape, device=DEV, dtype=I32)


def test_chunk_attention_and_append():
    P, Hq, Hkv, d, T, B, M = 6, 4, 2, 64, 3, 2, 4
    h = sas.sas_chunk_create(B, Hq, Hkv, d, M, P, T)
    Q, K, table, cu, kv = _bf(T, Hq, d), _bf(P, Hkv, 64, d), _ints(B, M), torch.tensor([0, 1, 3], device=DEV, dtype=I32), _ints(B) + 2

    def attention(Q=Q, K=K, V=K, table=table, O=None, LSE=None):
        sas.sas_chunk_attention(h, Q, K, V, table, cu, kv, torch.empty_like(Q) if O is None else O, LSE)

    attention()
    for bad in (_bf(T, Hq + 1, d), _bf(T, Hq // 2, d), _bf(T, Hq, 128), _bf(T, Hq * d)):
        with pytest.raises(ValueError, match="Q must have shape"):
            attention(Q=bad)
    for bad in (_bf(P - 1, Hkv, 64, d), _bf(P, 1, 64, d), _bf(P, Hkv, 32, d), _bf(P, Hkv, 64, 128)):
        with pytest.raises(ValueError, match="K_cache must have shape"):
            attention(K=bad, V=bad)
        with pytest.raises(ValueError, match="V_cache must have shape"):
            attention(V=bad)
    for bad in (_ints(B, M - 1), _ints(B, M + 1), _ints(B - 1, M)):
        with pytest.raises(ValueError, match="columns"):
            attention(table=bad)
    with pytest.raises(ValueError, match="O must have shape"):
        attention(O=_bf(T - 1, Hq, d))

    qkv, w, cos = _bf(T, Hq + 2 * Hkv, d), _bf(d), torch.ones(8, d // 2, device=DEV)
    pos, slots = _ints(T), torch.arange(T, device=DEV)

    def append(qkv=qkv, Q=Q, K=K, V=K):
        sas.sas_chunk_append(h, qkv, w, w, cos, cos, pos, slots, Q, K, V)

    V = torch.empty_like(K)
    append(V=V)
    for bad in (_bf(T, Hq - 1, d), _bf(T, Hq, 128), _bf(T - 1, Hq, d)):
        with pytest.raises(ValueError, match="Q must have shape|qkv must have shape"):
            append(Q=bad)
    for bad in (_bf(P - 1, Hkv, 64, d), _bf(P, 1, 64, d)):
        with pytest.raises(ValueError, match="cache must have shape"):
            append(K=bad, V=bad)
        with pytest.raises(ValueError, match="V_cache must have shape"):
            append(V=bad)
    with pytest.raises(ValueError, match="qkv must have shape"):
        append(qkv=_bf(T, Hq + 2, d))
    assert sas.sas_chunk_launch_count(h) == 3     # one attention (two kernels), one append
    assert sas.sas_chunk_get_device_status(h) == sas.SAS_OK
    sas.sas_chunk_destroy(h)


def test_norm_rope_and_its_gradient():
    B, N, H, Hkv, d = 2, 5, 4, 2, 64
    h = sas.sas_create(B, H, N, d, 0, Hkv=Hkv)
    qkv, w, cos = _bf(B, N, H + 2 * Hkv, d), _bf(d), torch.ones(N, d // 2, device=DEV)
    Q, K, dw = _bf(B, H, N, d), _bf(B, Hkv, N, d), torch.empty(2, d, device=DEV)
    V = torch.empty_like(K)
    sas.sas_qk_norm_rope_fwd(h, qkv, w, w, cos, cos, Q, K, V)
    sas.sas_qk_norm_rope_bwd(h, qkv, w, w, cos, cos, Q, K, V, torch.empty_like(qkv), dw[0], dw[1])
    n = sas.sas_launch_count(h)
    # all tensors of one smaller problem, which the library would take for its own
    small = dict(B=1, N=N, H=H, Hkv=Hkv), dict(B=B, N=N - 1, H=H, Hkv=Hkv), dict(B=B, N=N, H=2, Hkv=Hkv), dict(B=B, N=N, H=H, Hkv=1)
    for s in small:
        q, k = _bf(s["B"], s["H"], s["N"], d), _bf(s["B"], s["Hkv"], s["N"], d)
        x = _bf(s["B"], s["N"], s["H"] + 2 * s["Hkv"], d)
        with pytest.raises(ValueError, match="must have shape"):
            sas.sas_qk_norm_rope_fwd(h, x, w, w, cos, cos, q, k, torch.empty_like(k))
        with pytest.raises(ValueError, match="must have shape"):
            sas.sas_qk_norm_rope_bwd(h, x, w, w, cos, cos, q, k, k, torch.empty_like(x), dw[0], dw[1])
        with pytest.raises(ValueError, match="must have shape"):
            sas.sas_qk_norm_rope_fwd(h, qkv, w, w, cos, cos, q, k, torch.empty_like(k))
    assert sas.sas_launch_count(h) == n and sas.sas_get_device_status(h) == sas.SAS_OK
    sas.sas_destroy(h)
