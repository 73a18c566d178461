"""Every token of a warp's ring is turned by its own cosines and sines, the first ones included."""
import pytest
import torch

from paper_2609_13141_gb300 import sas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _turned(x, rot, inter):
    """x turned by a right angle: (a, b) -> (-b, a) in every pair."""
    y = x.clone()
    if inter:
        y[..., 0:rot:2], y[..., 1:rot:2] = -x[..., 1:rot:2], x[..., 0:rot:2]
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = -x[..., rot // 2:rot], x[..., :rot // 2]
    return y


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", [(8, 2, 128, 128), (8, 2, 128, 64), (4, 4, 64, 64), (4, 4, 64, 16)])
def test_right_angles_are_exact_from_the_first_token_on(Hq, Hkv, d, rot, inter):
    # cosines 0 and sines 1 permute the unturned outputs without any rounding; a warp has few tokens in every launch, so
    # that most are the first of their ring's stages
    N = 400
    g = torch.Generator(device=DEV)
    g.manual_seed(rot)
    qkv = torch.randn(1, N, Hq + 2 * Hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.randn(d, generator=g, device=DEV).to(torch.bfloat16)
    one, zero = torch.ones(N, rot // 2, device=DEV), torch.zeros(N, rot // 2, device=DEV)
    layer = sas.SasLayer(1, Hq, N, d, 0, Hkv=Hkv)
    Q0, K0, V0 = layer.qk_norm_rope(qkv, w, w, one, zero, interleaved=inter)
    dy = [torch.randn(*t.shape, generator=g, device=DEV).to(torch.bfloat16) for t in (Q0, K0, V0)]
    turned = (_turned(dy[0], rot, inter), _turned(dy[1], rot, inter), dy[2])
    want = layer.qk_norm_rope_bwd(qkv, w, w, one, zero, *dy, interleaved=inter)
    for _ in range(50):
        Q, K, V = layer.qk_norm_rope(qkv, w, w, zero, one, interleaved=inter)
        assert torch.equal(Q, _turned(Q0, rot, inter)) and torch.equal(K, _turned(K0, rot, inter)) and torch.equal(V, V0)
        # the transposed turn takes the turned gradient back to the unturned one's
        got = layer.qk_norm_rope_bwd(qkv, w, w, zero, one, *turned, interleaved=inter)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert sas.sas_get_device_status(layer.h) == sas.SAS_OK
    layer.close()
