"""What autograd follows is not passed by in silence: the calls around a step refuse it, before they look at anything else (so without a GPU)."""
import ctypes

import pytest
import torch
from torch.autograd import forward_ad

from paper_2603_19133_b200.binding import Context


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    ps.lib()
    c = Context.__new__(Context)
    c._h, c.device = ctypes.c_void_p(), 0
    return c


def _calls(ctx, x, one, g):
    """Each call with one tensor in one place, by name."""
    rows, K = torch.zeros(1, 1, 8), torch.zeros(1, 1, dtype=torch.int32)
    count = torch.zeros(1, dtype=torch.int32)
    return {"logits": lambda: ctx.penalize(x), "out": lambda: ctx.penalize(rows, out=x), "repetition": lambda: ctx.penalize(rows, repetition=one),
            "presence": lambda: ctx.penalize(rows, presence=one), "frequency": lambda: ctx.penalize(rows, frequency=one),
            "bias": lambda: ctx.penalize(rows, bias=(K, one.view(1, 1), count)),
            "grad": lambda: ctx.penalize_grad(x, rows), "grad's out": lambda: ctx.penalize_grad(rows, rows, out=x),
            "grad's repetition": lambda: ctx.penalize_grad(rows, rows, repetition=one), "grad's bias": lambda: ctx.penalize_grad(rows, rows, bias=(K, one.view(1, 1), count)),
            "norm": lambda: ctx.grad_norm([g]), "norm's out": lambda: ctx.grad_norm([], out=one), "clipped into others": lambda: ctx.clip_grad([g], 1.0, out=[rows]),
            "clip's norm": lambda: ctx.clip_grad([], 1.0, norm=one)}


def _refused_as_followed(call, name):
    with pytest.raises(Exception) as e:         # (where it is not: there is no GPU behind the tensors)
        call()
    return isinstance(e.value, ValueError) and "autograd" in str(e.value)


def test_what_requires_a_gradient_is_refused(ctx):
    x, one = torch.zeros(1, 1, 8, requires_grad=True), torch.ones(1, requires_grad=True)
    for name, call in _calls(ctx, x, one, 2 * x).items():
        assert _refused_as_followed(call, name), name
        with torch.no_grad():
            assert not _refused_as_followed(call, name), name
    for name, call in _calls(ctx, x.detach(), one.detach(), x.detach()).items():
        assert not _refused_as_followed(call, name), name


def test_a_leaf_has_a_norm_and_signs_are_read(ctx):
    x = torch.zeros(1, 1, 8, requires_grad=True)
    for call in (lambda: ctx.grad_norm([x]), lambda: ctx.penalize_grad(x.detach(), x), lambda: ctx.clip_grad([x], 1.0, out=[x.detach()])):
        assert not _refused_as_followed(call, "")


class Stand(Context):
    def __init__(self):
        pass

    def penalize(self, logits, *rules, **more):
        return logits.detach()


def test_a_tangent_of_forward_mode_is_refused(ctx):
    with forward_ad.dual_level():
        x, one = (forward_ad.make_dual(t, torch.ones_like(t)) for t in (torch.zeros(1, 1, 8), torch.ones(1)))
        for name, call in _calls(ctx, x, one, x).items():
            assert _refused_as_followed(call, name), name
        for call in (lambda: Stand().penalized(x), lambda: Stand().penalized(torch.zeros(1, 1, 8), repetition=one)):
            with pytest.raises(RuntimeError):
                call()
