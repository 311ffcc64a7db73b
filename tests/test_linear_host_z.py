"""What a kept pre-activation carries, and which gradients are refused without it (CPU only: nothing reaches a kernel)."""
import copy
import io

import pytest
import torch

from paper_2607_07386_amd import sdm


def kept():
    wide = torch.randn(2, 5, 12)
    z = wide.to(torch.bfloat16).as_subclass(sdm.Preactivation)
    z.rest = (wide - wide.to(torch.bfloat16).float()).to(torch.bfloat16)
    return wide, z


def test_widened_it_is_the_value_that_was_kept():
    wide, z = kept()
    rounded = wide.to(torch.bfloat16)
    for got in (z.float(), z.double(), z.to(torch.float32), z.to(dtype=torch.float64)):
        assert type(got) is torch.Tensor
        assert ((got.double() - wide.double()).abs() <= 2.0 ** -16 * wide.double().abs()).all()
    # narrow, it is the rounded value, and what torch makes of it is a plain tensor
    for got in (z + 0, z.clone(), z[:1], z.detach(), torch.cat([z, z]), z.to(torch.bfloat16, copy=True)):
        assert type(got) is torch.Tensor and got.dtype == torch.bfloat16
    assert torch.equal(z.to(torch.int32), rounded.to(torch.int32)) and torch.equal(z.to(torch.bool), rounded.to(torch.bool))
    assert torch.equal(z.clone(), rounded) and z.dtype == torch.bfloat16 and z.shape == (2, 5, 12)


def test_copied_or_saved_whole_it_keeps_the_rest():
    _, z = kept()
    f = io.BytesIO()
    torch.save(z, f)
    f.seek(0)
    loaded = torch.load(f, weights_only=False)      # this test's own bytes
    for got in (copy.copy(z), copy.deepcopy(z), loaded):
        assert type(got) is sdm.Preactivation and torch.equal(got.rest, z.rest) and torch.equal(got.clone(), z.clone())

    class Saves(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            ctx.save_for_backward(z)
            return x * 2

        @staticmethod
        def backward(ctx, g):
            assert type(ctx.saved_tensors[0]) is sdm.Preactivation and torch.equal(ctx.saved_tensors[0].rest, z.rest)
            return g * 2

    Saves.apply(torch.ones(3, requires_grad=True)).sum().backward()


def args(**kw):
    b = torch.bfloat16
    a = dict(x=torch.zeros(2, 5, 16, dtype=b), w=torch.zeros(12, 16, dtype=b), dy=torch.zeros(2, 5, 12, dtype=b), act=1,
             want_dbias=True)
    a.update(kw)
    return a


def test_dbias_without_the_rest_is_refused():
    _, z = kept()
    for plain in (z.clone(), z.detach(), torch.zeros(2, 5, 12, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="rounding left"):
            sdm.linear_bwd(**args(z=plain))


def test_what_keeps_enough_reaches_the_placement_check():
    _, z = kept()
    plain = z.clone()
    for kw in (dict(z=z), dict(z=plain, z_rest=z.rest), dict(z=plain.float()), dict(z=plain, want_dbias=False),
               dict(z=plain, act=0), dict(act=0)):
        with pytest.raises(ValueError, match="on the GPU"):
            sdm.linear_bwd(**args(**kw))
