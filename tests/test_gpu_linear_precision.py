"""How many bits the projections keep: the bias's gradient of the plain training call.

Tolerances count half steps (bf16 2^-8, fp32 2^-24).  A kept bf16 pre-activation with what its rounding left is off by
2^-16 of itself; |z act''(z)| < 1 for both activations, so a term of dbias is off by 2^-16 of dy at most, and their sum,
whose terms have either sign, by 2^-16 of its largest value and by the fp32 additions' sqrt(M) 2^-24."""
import pytest
import torch

from paper_2607_07386_amd import sdm
from tests.gpu_util import DEV
from tests.test_gpu_linear import ACTS, case, close, flat, reference

pytestmark = pytest.mark.gpu


def definition_gradients(x, w, bias, dy, act, hin, hout):
    """dx, dw, dbias of the definition in 64 bits, at its own unrounded pre-activation; and the pre-activation."""
    _, rz = reference(x.double(), w.double(), bias.double(), act, None, hout)
    zd = flat(rz).detach().requires_grad_()
    dz, = torch.autograd.grad(ACTS[act](zd), zd, flat(dy.double()))
    dz = dz.flatten(0, 1)
    dx = (dz @ w.double()).view(*flat(x).shape)
    dx = dx.unflatten(-1, (hin, -1)).transpose(1, 2) if hin else dx
    return dx, dz.T @ flat(x.double()).flatten(0, 1), dz.sum(0), rz


@pytest.mark.parametrize("act", [1, 2])
@pytest.mark.parametrize("kind", ["bf16", "bf16_dy_f32"])
@pytest.mark.parametrize("shape", [(3, 40, 64, 48, 0, 0), (2, 700, 40, 33, 0, 11), (1, 5, 64, 64, 4, 8), (4, 1, 128, 96, 0, 4),
                                   (2, 1500, 256, 192, 0, 6)])
def test_bias_gradient_of_the_plain_call(shape, kind, act):
    """y, z = linear(want_z) and linear_bwd(z=z): dbias is the unrounded definition's, z typed as y."""
    B, T, K, N, hin, hout = shape
    x, w, bias, _, dy = case(B, T, K, N, hin, hout, True)
    dy = dy.float() * 1.001 if kind == "bf16_dy_f32" else dy
    y, z = sdm.linear(x, w, bias, act=act, heads=hout, want_z=True)
    assert z.dtype == y.dtype == torch.bfloat16
    g = sdm.linear_bwd(x, w, dy, z=z, act=act, want_dbias=True)
    _, _, dbias, _ = definition_gradients(x, w, bias, dy, act, hin, hout)
    close(g["dbias"], dbias, "dbias", 2.0 ** -16 + (B * T) ** 0.5 * 2.0 ** -24)
    # alone, or with what the rounding left handed over beside z, the same sum
    assert torch.equal(sdm.linear_bwd(x, w, dy, z=z, act=act, want_dx=False, want_dw=False, want_dbias=True)["dbias"],
                       g["dbias"])
    _, z2, rest = sdm.linear(x, w, bias, act=act, heads=hout, want_z=True, want_rest=True)
    g2 = sdm.linear_bwd(x, w, dy, z=z2, z_rest=rest, act=act, want_dbias=True)
    for name in g:
        assert torch.equal(g[name], g2[name]), name

