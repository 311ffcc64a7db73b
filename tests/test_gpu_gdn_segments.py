"""The dense rule's segments side by side against the definition in 64 bits, with several column tiles to a workgroup.
Tolerance: see tests/test_gpu_gdn.py."""
import pytest
import torch

from paper_2607_07386_amd import sdm
from tests.gpu_util import DEV
from tests.test_gpu_gdn import close, definition, inputs

pytestmark = pytest.mark.gpu


# On 256 compute units 512 column tiles of the segments' ends (of d_v and d_k, without the last segment) put two tiles
# to a workgroup, 1024 four, where the kernel has that form.  d_v = 100 has seven tiles: a workgroup holds columns of
# values and of the multiplier side by side.
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Hk,H,dk,dv", [
    (24, 1, 1, 128, 100),       # 1440 tiles: four (bf16), two (fp32)
    (12, 1, 1, 128, 100),       # 720: two
    (24, 1, 1, 64, 100),        # 1056: four in either type
    (4, 2, 6, 128, 128),        # three value heads to a key head
    (3, 1, 2, 256, 36),
])
def test_values_of_segments_side_by_side(B, Hk, H, dk, dv, bf16):
    T = 5 * 16 * 64 + 130
    a, s0, _, _ = inputs(B, Hk, H, T, dk, dv, bf16, seed=11, long_memory=True)
    lens = torch.tensor([T, 3333, 50, 0][:B] + [T - 64 * b for b in range(4, B)], dtype=torch.int32, device=DEV)
    on = (torch.arange(T, device=DEV)[None] < lens[:, None])[:, None, :, None]
    ry, rS = definition(a, s0, lens)
    y, S = sdm.gdn_fwd(**a, state0=s0, lens=lens)
    close(torch.where(on, y, 0.0), ry, "y")
    close(S, rS, "state")
    saved = sdm.gdn_saved_buffer(B, H, T, dk, dv, torch.device(DEV))
    y2, S2 = sdm.gdn_fwd(**a, state0=s0, lens=lens, saved=saved)
    assert torch.equal(torch.where(on, y, 0.0), torch.where(on, y2, 0.0)) and torch.equal(S, S2)
