"""Refusals of the projections (CPU only: nothing reaches a kernel)."""
import pytest
import torch

from paper_2607_07386_amd import sdm

L = sdm.lib()
A = 0x10000000    # aligned, compared but never used
BIG = 1 << 40


def fwd(**kw):
    a = dict(x=A, xd=1, xh=0, w=A, wd=1, bias=None, act=0, res=None, B=2, T=300, K=64, N=96, yh=0, y=A, yd=1, z=None,
             rest=None, ws=A, wsb=BIG)
    a.update(kw)
    return L.sdm_linear(*a.values(), None)


def bwd(**kw):
    a = dict(x=A, xd=1, xh=0, w=A, wd=1, z=A, rest=None, zd=1, act=1, dy=A, dyd=1, B=2, T=300, K=64, N=96, yh=0, dx=A, dw=A,
             db=A, ws=A, wsb=BIG)
    a.update(kw)
    return L.sdm_linear_bwd(*a.values(), None)


SIZES = [(dict(B=-1), -1), (dict(T=-1), -1), (dict(K=0), -1), (dict(N=0), -1), (dict(K=60), -1), (dict(K=66), -1),
         (dict(xd=2), -1), (dict(wd=-1), -1), (dict(wd=0), -1), (dict(act=3), -1), (dict(act=-1), -1), (dict(xh=3), -1),
         (dict(xh=16), -1), (dict(yh=7), -1), (dict(xh=-1), -1), (dict(yh=-1), -1), (dict(B=1 << 20, T=1 << 20), -2), (dict(B=1 << 13, T=(1 << 13) + 1), -2),
         (dict(K=(1 << 24) + 8), -2), (dict(N=(1 << 22) + 1), -2), (dict(x=None), -1), (dict(w=None), -1),
         (dict(x=A + 8), -1), (dict(w=A + 2), -1)]


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(y=None), -1), (dict(y=A + 8), -1), (dict(z=A + 4), -1), (dict(res=A + 2), -1), (dict(rest=A), -1), (dict(z=A, rest=A + 4), -1), (dict(z=A, rest=A, yd=0), -1), (dict(bias=A + 2), -1),
    (dict(yd=2), -1), (dict(xd=0, wd=0, yd=1), -1), (dict(res=A, yh=8), -1),
    (dict(xd=0, wd=0, yd=0, ws=None), -1), (dict(xd=0, wd=0, yd=0, wsb=16), -3)])
def test_forward_refuses(kw, code):
    assert fwd(**kw) == code
    assert L.sdm_last_error()


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(z=None), -1), (dict(dy=None), -1), (dict(dy=A + 8), -1), (dict(dx=A + 8), -1), (dict(dw=A + 8), -1),
    (dict(db=A + 2), -1), (dict(zd=3), -1), (dict(dyd=3), -1), (dict(rest=A, zd=0), -1), (dict(rest=A + 8), -1), (dict(xd=0, wd=0, dyd=1, zd=0), -1),
    (dict(xd=0, wd=0, dyd=0, zd=1), -1), (dict(ws=None), -1), (dict(wsb=100), -3), (dict(ws=A + 64), -1)])
def test_backward_refuses(kw, code):
    assert bwd(**kw) == code
    assert L.sdm_last_error()


def test_nothing_to_do():
    assert fwd(B=0) == 0 and fwd(T=0) == 0
    assert bwd(dx=None, dw=None, db=None) == 0


def _t(*s, dt=torch.float32):
    return torch.zeros(s, dtype=dt)


@pytest.mark.parametrize("kw", [
    dict(x=_t(5, 16)), dict(x=_t(2, 5, 24)), dict(w=_t(12, 16).double()), dict(x=_t(2, 5, 16, dt=torch.bfloat16)),
    dict(bias=_t(11)), dict(bias=_t(12, dt=torch.bfloat16)), dict(residual=_t(2, 5, 16)), dict(heads=5), dict(heads=-1),
    dict(residual=_t(2, 5, 12), heads=3), dict(out_dtype=torch.bfloat16), dict(out_dtype=torch.float16),
    dict(y=_t(2, 5, 13)), dict(y=_t(2, 3, 5, 4)), dict(workspace=_t(4)), dict(x=[1]), dict(want_rest=True)])
def test_binding_refuses(kw):
    a = dict(x=_t(2, 5, 16), w=_t(12, 16))
    a.update(kw)
    with pytest.raises((ValueError, TypeError)) as e:
        sdm.linear(**a)
    assert "GPU" not in str(e.value)


@pytest.mark.parametrize("kw", [
    dict(dy=_t(2, 5, 16)), dict(dy=_t(2, 6, 12)), dict(dy=_t(2, 5, 12).double()), dict(act=1),
    dict(act=1, z=_t(2, 3, 5, 4)), dict(z=_t(2, 5, 12).double()), dict(z_rest=_t(2, 5, 12, dt=torch.bfloat16)),
    dict(z=_t(2, 5, 12), z_rest=_t(2, 5, 12, dt=torch.bfloat16)), dict(workspace=torch.zeros(1, dtype=torch.uint8))])
def test_binding_refuses_backward(kw):
    a = dict(x=_t(2, 5, 16), w=_t(12, 16), dy=_t(2, 5, 12))
    a.update(kw)
    with pytest.raises((ValueError, TypeError)) as e:
        sdm.linear_bwd(**a)
    assert "GPU" not in str(e.value)


def test_good_arguments_reach_the_placement_check():
    for x in (_t(2, 5, 16), _t(2, 4, 5, 4)):
        with pytest.raises(ValueError, match="on the GPU"):
            sdm.linear(x, _t(12, 16), _t(12), act=1, heads=3, want_z=True)
