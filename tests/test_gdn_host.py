"""Refusals of the dense gated delta rule (CPU only: nothing reaches a kernel)."""
import pytest
import torch

from paper_2607_07386_amd import sdm

L = sdm.lib()
A = 0x10000000    # 256-byte aligned, compared but never used
BIG = 1 << 40


def fwd(**kw):
    a = dict(q=A, k=A, v=A, dt=1, al=A, be=A, lens=None, s0=None, sT=A, B=2, Hk=2, H=4, T=100, dk=64, dv=64, y=A,
             saved=None, sb=0, ws=A, wsb=BIG)
    a.update(kw)
    return L.sdm_gdn_fwd(*a.values(), None)


def bwd(**kw):
    a = dict(q=A, k=A, v=A, dt=1, al=A, be=A, lens=None, saved=A, sb=BIG, dy=A, dsT=None, B=2, Hk=2, H=4, T=100, dk=64,
             dv=64, dq=A, dkk=A, dvv=A, dal=A, dbe=A, ds0=None, ws=A, wsb=BIG)
    a.update(kw)
    return L.sdm_gdn_bwd(*a.values(), None)


SIZES = [(dict(H=3), -1), (dict(Hk=0), -1), (dict(H=0), -1), (dict(B=-1), -1), (dict(T=-1), -1), (dict(dk=6), -1),
         (dict(dk=0), -1), (dict(dv=2), -1), (dict(dk=260), -2), (dict(dv=4100), -2), (dict(B=20000), -2),
         (dict(T=(1 << 30) + 1), -2), (dict(dt=2), -1), (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1),
         (dict(al=None), -1), (dict(be=None), -1), (dict(q=A + 8), -1), (dict(v=A + 4), -1), (dict(lens=A + 2), -1),
         (dict(ws=None), -1), (dict(ws=A + 16), -1), (dict(wsb=1000), -3)]


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(sT=None), -1), (dict(sT=A + 4), -1), (dict(s0=A + 4), -1), (dict(y=None), -1), (dict(y=A + 8), -1),
    (dict(saved=A, sb=100), -3), (dict(saved=A + 16, sb=BIG), -1)])
def test_forward_refuses(kw, code):
    assert fwd(**kw) == code
    assert L.sdm_last_error()


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(saved=None), -1), (dict(sb=100), -3), (dict(dy=None), -1), (dict(dq=None), -1), (dict(dkk=None), -1),
    (dict(dvv=None), -1), (dict(dal=None), -1), (dict(dbe=None), -1), (dict(dy=A + 4), -1), (dict(dsT=A + 4), -1),
    (dict(ds0=A + 4), -1), (dict(dal=A + 2), -1)])
def test_backward_refuses(kw, code):
    assert bwd(**kw) == code
    assert L.sdm_last_error()


def test_nothing_to_do():
    assert fwd(B=0) == 0 and bwd(B=0) == 0


def test_sizes():
    assert L.sdm_gdn_fwd_workspace_bytes(4, 2, 2, 1, 64, 64, 1, 0) == 0      # the decode step needs none
    assert L.sdm_gdn_fwd_workspace_bytes(4, 2, 2, 4096, 64, 64, 1, 0) > 0
    assert L.sdm_gdn_fwd_workspace_bytes(4, 2, 2, 1, 64, 64, 1, 1) > 0
    # one state per 64 tokens and one row per token
    assert L.sdm_gdn_saved_bytes(2, 4, 100, 64, 32) == 2 * 4 * (2 * 64 * 32 + 100 * 32) * 4
    assert L.sdm_gdn_saved_bytes(2, 4, 100, 63, 32) == 0


def _args(**kw):
    B, Hk, H, T, dk, dv = 2, 2, 4, 5, 8, 12
    z = torch.zeros
    a = dict(q=z(B, Hk, T, dk), k=z(B, Hk, T, dk), v=z(B, H, T, dv), alpha=z(B, H, T), beta=z(B, H, T))
    a.update(kw)
    return a


@pytest.mark.parametrize("kw", [
    dict(q=torch.zeros(2, 2, 5)), dict(k=torch.zeros(2, 2, 5, 12)), dict(k=torch.zeros(2, 2, 5, 8).bfloat16()),
    dict(q=torch.zeros(2, 2, 5, 8).double()), dict(v=torch.zeros(2, 3, 5, 12)), dict(v=torch.zeros(2, 4, 6, 12)),
    dict(alpha=torch.zeros(2, 4, 4)), dict(beta=torch.zeros(2, 4, 5).bfloat16()), dict(lens=torch.zeros(2)),
    dict(lens=torch.zeros(3, dtype=torch.int32)), dict(state0=torch.zeros(2, 4, 12, 8)),
    dict(state_out=torch.zeros(2, 4, 8, 12).bfloat16()), dict(y=torch.zeros(2, 4, 5, 8)),
    dict(saved=torch.zeros(16, dtype=torch.uint8)), dict(workspace=torch.zeros(64)),
])
def test_binding_refuses(kw):
    with pytest.raises((ValueError, TypeError)) as e:
        sdm.gdn_fwd(**_args(**kw))
    assert "GPU" not in str(e.value)


@pytest.mark.parametrize("kw", [dict(dy=torch.zeros(2, 4, 5, 8)), dict(dy=torch.zeros(2, 4, 5, 12).bfloat16()),
                                dict(dstate_T=torch.zeros(2, 4, 8, 8)), dict(saved=None),
                                dict(saved=torch.zeros(8, dtype=torch.uint8))])
def test_binding_refuses_backward(kw):
    a = _args(saved=torch.zeros(sdm.lib().sdm_gdn_saved_bytes(2, 4, 5, 8, 12), dtype=torch.uint8),
              dy=torch.zeros(2, 4, 5, 12))
    a.update(kw)
    with pytest.raises((ValueError, TypeError)) as e:
        sdm.gdn_bwd(**a)
    assert "GPU" not in str(e.value)


def test_good_arguments_reach_the_placement_check():
    with pytest.raises(ValueError, match="on the GPU"):
        sdm.gdn_fwd(**_args())
