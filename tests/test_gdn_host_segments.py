"""Where the dense rule runs segments of the sequence side by side (CPU only): their states are part of the workspace."""
import pytest

from paper_2607_07386_amd import sdm

L = sdm.lib()


def segmented(B, Hk, H, T, dk, dv, bf16):
    n = B * H * ((T + 63) // 64)
    up = lambda x: (x + 255) // 256 * 256
    one = up(n * 6 * 64 * 4) + 2 * up(n * 6 * 3 * 512 * 2)        # per chunk: six vectors, fragments of T' and P
    have = L.sdm_gdn_fwd_workspace_bytes(B, Hk, H, T, dk, dv, int(bf16), 0)
    assert have >= one
    return have > one


@pytest.mark.parametrize("B,H,T,dk,dv,bf16", [
    (1, 16, 65536, 128, 128, True), (1, 1, 5120, 64, 64, True), (1, 24, 16384, 128, 128, False),
    (1, 4, 16384, 256, 256, False), (1, 16, 16384, 128, 64, True), (1, 48, 16384, 64, 16, True)])
def test_where_segments_were_measured_faster(B, H, T, dk, dv, bf16):
    assert segmented(B, H, H, T, dk, dv, bf16)


@pytest.mark.parametrize("B,H,T,dk,dv,bf16", [
    (1, 24, 5120, 256, 128, False), (1, 16, 5120, 256, 128, False), (1, 24, 65536, 256, 128, False),   # 1.45, 1.20, 1.37
    (1, 204, 5120, 256, 16, False), (1, 100, 16384, 256, 32, False), (1, 50, 16384, 256, 64, False),   # 3.24, 2.36, 1.79
    (1, 204, 16384, 64, 16, True), (1, 100, 16384, 128, 16, True), (1, 24, 5120, 256, 128, True)])     # 1.61, 1.35, 1.06
def test_where_segments_were_measured_slower(B, H, T, dk, dv, bf16):
    assert not segmented(B, H, H, T, dk, dv, bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Hk,H,T,dk,dv", [
    # the shapes of the GPU tests of segments: tests/test_gpu_gdn.py, tests/test_gpu_gdn_segments.py
    (4, 1, 1, 5820, 16, 20), (4, 1, 1, 5820, 128, 48), (4, 1, 1, 5820, 132, 20), (4, 1, 1, 5820, 256, 36),
    (24, 1, 1, 5120, 128, 128), (24, 1, 1, 5250, 128, 100), (12, 1, 1, 5250, 128, 100), (24, 1, 1, 5250, 64, 100), (4, 2, 6, 5250, 128, 128),
    (3, 1, 2, 5250, 256, 36)])

def test_the_tests_of_segments_have_them(B, Hk, H, T, dk, dv, bf16):
    assert segmented(B, Hk, H, T, dk, dv, bf16)
