"""Which tile and which split of the depth the large calls of tests/test_gpu_linear_tiles.py take (CPU only)."""
import ctypes

import pytest

from paper_2607_07386_amd import sdm

plan_fn = sdm.lib()._Z15sdm_linear_planiii      # LinPlan sdm_linear_plan(int I, int J, int steps): {bool big; int split}
plan_fn.restype = ctypes.c_uint64

# B, T, K, N, heads in, heads out, bf16: between them 256 x 256 tiles in each direction, with depths that are whole
# multiples of 64 and others, split and not; fp32 factors stand as padded parts, so theirs are always whole
LARGE = [(1, 4099, 1032, 2000, 0, 0, True), (2, 2048, 1032, 2000, 0, 25, True), (2, 2050, 2000, 1000, 50, 0, True),
         (1, 4096, 2048, 1024, 32, 16, True), (1, 2000, 8200, 1030, 0, 0, True), (1, 2048, 8192, 1088, 0, 17, True),
         (1, 2000, 1032, 8200, 0, 0, True), (1, 2048, 1024, 8192, 0, 64, True), (1, 4099, 1032, 2000, 0, 0, False),
         (2, 1025, 1032, 1000, 129, 8, False)]


def plan(I, J, steps):
    p = plan_fn(I, J, steps)
    return bool(p & 0xff), p >> 32


def taken(B, T, K, N, hin, hout, bf16):
    """{direction: (256 x 256 tile, depth in whole steps of 64, split)}, as linear_api.cpp and even_depth choose."""
    M, combos = B * T, 1 if bf16 else 6
    whole = dict(fwd=K % 64 == 0 and (not hin or K // hin % 64 == 0), dx=N % 64 == 0,
                 dw=(M if not hin or B == 1 else T) % 64 == 0)
    sizes = dict(fwd=(M, N, K), dx=(M, K, N), dw=(N, K, M))
    out = {}
    for way, (I, J, R) in sizes.items():
        big, split = plan(I, J, (R + 63) // 64 * combos)
        out[way] = (big, whole[way] or not bf16, split > 1)
    return out


@pytest.mark.parametrize("way", ["fwd", "dx", "dw"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("split", [True, False])
def test_every_large_tile_is_reached(way, whole, split):
    assert (True, whole, split) in [taken(*c)[way] for c in LARGE if c[-1]]


@pytest.mark.parametrize("way", ["fwd", "dx", "dw"])
def test_large_tiles_of_fp32_parts_are_reached(way):
    assert any(taken(*c)[way][0] for c in LARGE if not c[-1])
