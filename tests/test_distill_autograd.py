"""What Context.distill_loss tells autograd, without a GPU: the library's call is stood in for."""
import pytest
import torch

from paper_2603_19133_b200.binding import Context


class Stand(Context):
    """A context whose distill is sum over the vocabulary of logits squared."""

    def __init__(self):
        self.calls = []

    def distill(self, logits, temperature, t_idx, t_prob, t_count, weight=None, tail=False, want_loss=True, want_grad=True, out=None):
        self.calls.append((want_loss, want_grad))
        loss = (logits.detach() ** 2).sum(-1) if want_loss else None
        return loss, 2 * logits.detach() * (1.0 if weight is None else weight[..., None]) if want_grad else None


def _inputs():
    return torch.randn(2, 3, 7), torch.ones(2), torch.zeros(2, 3, 1, dtype=torch.int32), torch.ones(2, 3, 1), torch.ones(2, 3, dtype=torch.int32)


def test_the_logits_get_the_gradient_for_the_weights_that_come():
    x, T, idx, t, n = _inputs()
    ctx, leaf, w = Stand(), x.clone().requires_grad_(True), torch.randn(2, 3)
    (ctx.distill_loss(leaf, T, idx, t, n) * w).sum().backward()
    torch.testing.assert_close(leaf.grad, 2 * x * w[..., None])
    assert ctx.calls == [(True, False), (False, True)]


@pytest.mark.parametrize("which", ["temperature", "t_prob"])
def test_inputs_without_a_gradient_are_refused_where_one_is_wanted(which):
    x, T, idx, t, n = _inputs()
    ctx, leaf = Stand(), x.clone().requires_grad_(True)
    (T if which == "temperature" else t).requires_grad_(True)
    for logits in (leaf, x):
        with pytest.raises(ValueError, match=which):
            ctx.distill_loss(logits, T, idx, t, n)
    # where none is wanted they are values like any other
    with torch.no_grad():
        assert not ctx.distill_loss(leaf, T, idx, t, n).requires_grad
    ctx.distill_loss(leaf, T.detach(), idx, t.detach(), n).sum().backward()
    assert leaf.grad is not None
