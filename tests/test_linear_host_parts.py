"""The tolerance of the fp32 projections' tests is below what the loss of one product of parts leaves (CPU only).

An fp32 value is cut into bf16 parts t0 + t1 + t2, each the top 16 bits of what is left; six products of parts, of
total order up to two, make a product.  Emulated in 64 bits."""
import numpy as np
import pytest

ORDER_2 = [(0, 2), (1, 1), (2, 0)]
KEPT = ORDER_2 + [(0, 1), (1, 0), (0, 0)]


def parts(x):
    out = []
    for _ in range(3):
        t = (x.astype(np.float32).view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        out.append(t.astype(np.float64))
        x = (x - t).astype(np.float32)      # exact
    return out


def f32_tol(depth):     # as tests/test_gpu_linear_precision.py has it
    return 2.0 ** -20 + depth ** 0.5 * 2.0 ** -24


@pytest.mark.parametrize("depth", [8, 64, 256, 704, 1024, 2000, 5000])
def test_a_lost_product_exceeds_the_tolerance(depth):
    rng = np.random.default_rng(depth)
    x, w = rng.standard_normal((200, depth)).astype(np.float32), rng.standard_normal((64, depth)).astype(np.float32)
    px, pw = parts(x), parts(w)
    exact = x.astype(np.float64) @ w.astype(np.float64).T
    error = lambda kept: np.abs(sum(px[i] @ pw[j].T for i, j in kept) - exact).max() / np.abs(exact).max()
    assert error(KEPT) < f32_tol(depth) / 4
    for lost in KEPT:
        assert error([p for p in KEPT if p != lost]) > f32_tol(depth), lost
