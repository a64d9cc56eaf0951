"""The calls around a step: what they record, allocate, hold on to and refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(1, 1, 200000, 1)
    yield c
    c.close()


def test_a_norm_is_recorded_as_a_norm(ctx):
    # 11: grad_norm, and clip_grad's pass over the squares; 12: the pass that scales, which grad_norm has none of
    g = torch.randn(5000, device="cuda")
    ctx.profile_enable(1)
    for _ in range(3):
        ctx.grad_norm([g])
    assert len(ctx.profile_samples(11)) == 3 and len(ctx.profile_samples(12)) == 0
    norm = ctx.grad_norm([g])
    for _ in range(2):
        ctx.clip_grad([g], 1.0)
    ctx.clip_grad([g], 1.0, norm=norm)
    assert len(ctx.profile_samples(11)) == 3 and len(ctx.profile_samples(12)) == 3
    ctx.profile_enable(0)
