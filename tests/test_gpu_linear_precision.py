"""How many bits the projections keep: the bias's gradient of the plain training call, fp32 operands beside bf16 ones.

Tolerances count half steps (bf16 2^-8, fp32 2^-24).  A kept bf16 pre-activation with what its rounding left is off by
2^-16 of itself; |z act''(z)| < 1 for both activations, so a term of dbias is off by 2^-16 of dy at most, and their sum,
whose terms have either sign, by 2^-16 of its largest value and by the fp32 additions' sqrt(M) 2^-24.  A product of fp32
parts leaves out terms of order 3 and above: the parts are cut, so each is below 2^-7 of the one before, and what is
left out below 2^-20 of the term; the sum of K terms adds sqrt(K) 2^-24 (roundings either way).  Two parts leave
2^-15 of a term.  A bf16 result is one half step off on top."""
import pytest
import torch

from paper_2607_07386_amd import sdm
from tests.gpu_util import DEV
from tests.test_gpu_linear import ACTS, SHAPES, case, close, flat, reference

pytestmark = pytest.mark.gpu

HALF_BF16 = 2.0 ** -8


def f32_tol(depth):
    return 2.0 ** -20 + depth ** 0.5 * 2.0 ** -24


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


MIXED = [  # B, T, K, N, heads in, heads out: few rows, few outputs, tiles, odd sizes, a split depth, large tiles
    (3, 1, 64, 40, 4, 0), (16, 1, 256, 512, 0, 4), (2, 200, 136, 24, 0, 0), (2, 257, 96, 96, 2, 3), (1, 300, 704, 260, 0, 0),
    (3, 50, 520, 90, 13, 0), (1, 640, 512, 512, 8, 8), (1, 129, 4096, 130, 0, 0), (1, 4099, 1032, 2000, 0, 0),
]


@pytest.mark.parametrize("shape", MIXED)
def test_fp32_rows_beside_bf16_weights(shape):
    """An fp32 x enters in full: an fp32 result to fp32's accuracy, a bf16 one off by its own rounding."""
    B, T, K, N, hin, hout = shape
    x, w, bias, _, _ = case(B, T, K, N, hin, hout, True, x_f32=True)
    ry, _ = reference(x.double(), w.double(), bias.double(), 0, None, hout)
    y, z = sdm.linear(x, w, bias, heads=hout, out_dtype=torch.float32, want_z=True)
    close(y, ry, "y in fp32", f32_tol(K))
    assert torch.equal(y, z)
    y = sdm.linear(x, w, bias, heads=hout)
    size, _ = reference(x.double().abs(), w.double().abs(), bias.double().abs(), 0, None, hout)
    over = (y.double() - ry).abs() - HALF_BF16 * ry.abs() - 2.0 ** -14 * size / K ** 0.5
    assert over.max() <= 0, f"a bf16 result is off by more than its rounding: {over.max():.2e}"


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("x_f32,dy_f32", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("shape", MIXED)
def test_gradients_of_fp32_rows_beside_bf16_weights(shape, x_f32, dy_f32, act):
    """An fp32 x or dy enters the gradients with more bits than a bf16 result keeps; an fp32 dx is one of fp32's accuracy."""
    B, T, K, N, hin, hout = shape
    x, w, bias, _, dy = case(B, T, K, N, hin, hout, True, x_f32=x_f32)
    dy = dy.float() * 1.001 if dy_f32 else dy
    z = None
    if act:
        _, z = sdm.linear(x, w, bias, act=act, heads=hout, want_z=True)
    g = sdm.linear_bwd(x, w, dy, z=z, act=act, want_dbias=True)
    dx, dw, dbias, _ = definition_gradients(x, w, bias, dy, act, hin, hout)
    # the slope's own place (the kept z, and an fp32 x that entered it in two parts), then the activation's roundings
    at_z = (2.0 ** -16 + (2.0 ** -15 if x_f32 else 0.0) + 2.0 ** -20) if act else 0.0
    close(g["dbias"], dbias, "dbias", at_z + 2.0 ** -24 + (B * T) ** 0.5 * 2.0 ** -24)
    if x_f32:
        close(g["dx"], dx, "dx", at_z + f32_tol(N))
    # two cut parts leave 2^-14 of a term, in a sum of either sign of its root mean square
    for name, ref in (("dw", dw),) if x_f32 else (("dx", dx), ("dw", dw)):
        over = (g[name].double() - ref).abs() - HALF_BF16 * ref.abs() - 2.0 ** -11 * ref.square().mean().sqrt()
        assert over.max() <= 0, f"{name} is off by more than its rounding: {over.max():.2e}"


@pytest.mark.parametrize("bf16", [True, False])
def test_bias_gradient_alone_writes_no_dz(bf16):
    """With neither dx nor dw wanted, dz's planes at the workspace's start are left as they were."""
    x, w, bias, _, dy = case(2, 300, 64, 96, 0, 6, bf16)
    _, z = sdm.linear(x, w, bias, act=1, heads=6, want_z=True)
    code = int(bf16)
    ws = torch.full((sdm.lib().sdm_linear_bwd_workspace_bytes(code, code, 1, code, 2, 300, 64, 96, 6),), 0xA5,
                    dtype=torch.uint8, device=DEV)
    g = sdm.linear_bwd(x, w, dy, z=z, act=1, want_dx=False, want_dw=False, want_dbias=True, workspace=ws)
    planes = (1 if bf16 else 3) * 640 * 128 * 2
    assert (ws[:planes] == 0xA5).all() and not (ws == 0xA5).all()
    assert torch.equal(g["dbias"], sdm.linear_bwd(x, w, dy, z=z, act=1, want_dbias=True)["dbias"])


@pytest.mark.parametrize("shape", SHAPES + [(1, 5000, 136, 16, 0, 0), (1, 3000, 72, 64, 0, 0), (1, 2000, 68, 33, 17, 3)])
def test_fp32_products_lose_no_part(shape):
    """All fp32, at a tolerance that the loss of any one product of parts exceeds up to 5,000 terms (tests/test_linear_host_parts.py)."""
    B, T, K, N, hin, hout = shape
    x, w, bias, _, dy = case(B, T, K, N, hin, hout, False)
    for act in (0, 1, 2):
        y, z = sdm.linear(x, w, bias, act=act, heads=hout, want_z=True)
        ry, rz = reference(x.double(), w.double(), bias.double(), act, None, hout)
        close(z, rz, "z", f32_tol(K))
        close(y, ry, "y", f32_tol(K) if act == 0 else 2 * f32_tol(K))     # a slope of at most 1.1, and its own roundings
    g = sdm.linear_bwd(x, w, dy, want_dbias=True)
    dx, dw, dbias, _ = definition_gradients(x, w, bias, dy, 0, hin, hout)
    close(g["dx"], dx, "dx", f32_tol(N))
    close(g["dw"], dw, "dw", f32_tol(B * T))
    close(g["dbias"], dbias, "dbias", f32_tol(B * T))
