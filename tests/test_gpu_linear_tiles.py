"""Projections large enough for 256 x 256 tiles, in each direction, whole and split depths, sizes that divide nothing.

Tolerances: see tests/test_gpu_linear_precision.py.  bf16 products are exact and their fp32 sums off by sqrt(n) 2^-24 of
the sum's own size for roundings either way, so a bf16 result is off by its own rounding and at most 2^-14 of the
results' root mean square (n <= 8,200: 2^-17); a wrong or missing term of any depth is 2^-7 of that or more."""
import pytest
import torch

from paper_2607_07386_amd import sdm
from tests.test_gpu_linear import case, flat, reference
from tests.test_gpu_linear_precision import HALF_BF16, close, f32_tol
from tests.test_linear_host_tiles import LARGE

pytestmark = pytest.mark.gpu


def rounded_once(got, ref, what):
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    over = (got.double() - ref).abs() - HALF_BF16 * ref.abs() - 2.0 ** -14 * ref.square().mean().sqrt()
    assert over.max() <= 0, f"{what}: {over.max():.2e} beyond its rounding"


@pytest.mark.parametrize("B,T,K,N,hin,hout,bf16", LARGE)
def test_large_tiles(B, T, K, N, hin, hout, bf16):
    x, w, bias, res, dy = case(B, T, K, N, hin, hout, bf16)
    near = rounded_once if bf16 else (lambda got, ref, what: close(got, ref, what, f32_tol(max(K, N, B * T))))
    rx, rw = x.double(), w.double()
    ry, _ = reference(rx, rw, None, 0, None, hout)
    near(sdm.linear(x, w, heads=hout), ry, "y")
    res = None if hout else res
    ry, rz = reference(rx, rw, bias.double(), 1, None if res is None else res.double(), hout)
    y, z = sdm.linear(x, w, bias, act=1, residual=res, heads=hout, want_z=True)
    near(z.clone(), rz, "z")
    if bf16:
        rounded_once(y, ry, "y of an activation")
    else:
        close(y, ry, "y of an activation", 2 * f32_tol(K))     # z times a slope of at most 1.1, and its own roundings
    del y, z, ry, rz
    g = sdm.linear_bwd(x, w, dy, want_dbias=True)
    dz = flat(dy.double()).flatten(0, 1)
    dx = (dz @ rw).view(B, T, K)
    near(g["dx"], dx.unflatten(-1, (hin, -1)).transpose(1, 2) if hin else dx, "dx")
    near(g["dw"], dz.T @ flat(rx).flatten(0, 1), "dw")
    close(g["dbias"], dz.sum(0), "dbias", f32_tol(B * T))
