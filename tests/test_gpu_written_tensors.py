"""The library's calls write into tensors behind torch's back; autograd has to hear of it, or a backward pass takes what was written later for
what it saved."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, G, V, K = 2, 3, 4000, 16


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(B, G + 1, V, K)
    yield c
    c.close()


def _rows(R=G, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((B, R, V), generator=g, device="cuda"), torch.ones(B, device="cuda"), torch.rand((B, R, 2), generator=g, device="cuda")


def test_every_call_raises_the_versions_of_its_outputs(ctx):
    draft, T, u2 = _rows()
    target = _rows(G + 1, 4)[0]
    u = u2[..., 0].contiguous()
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    q = ctx.compress(draft, T, K, 1.0, K, u)
    uv, ur = u2[..., 1].contiguous(), u2[:, 0].contiguous()
    args = (target, T, q[3], *q[:3], uv, ur)
    v = ctx.verify(*args)
    r = ctx.verify_range(target, T, None, 0, G + 1, None, q[3], *q[:3], uv, ur)
    top = ctx.target_topk(target, T, pos, K)
    e = ctx.edge_resample(draft, T, pos, *top, ur[:, 0].contiguous())
    s = ctx.residual_sample(target, T, pos, *q[:3], ur)
    buf, nbytes = ctx.wire_pack(*q[:3])
    w = ctx.wire_unpack(buf, int(nbytes.item()), B * G, K)
    d = ctx.distill(draft, T, *q[:3])
    t = ctx.sample(draft, T, u2)
    for call, outs in [
            (lambda: ctx.compress(draft, T, K, 1.0, K, u, out=q), q),
            (lambda: ctx.verify(*args, out=v), v.values()),
            (lambda: ctx.verify_range(target, T, None, 0, G + 1, None, q[3], *q[:3], uv, ur, out=r), r.values()),
            (lambda: ctx.target_topk(target, T, pos, K, out=top), top),
            (lambda: ctx.distill(draft, T, *q[:3], out=d), d),
            (lambda: ctx.sample(draft, T, u2, out=t), t)]:
        before = [x._version for x in outs]
        call()
        assert all(x._version > n for x, n in zip(outs, before))
        read = [x._version for x in (draft, target, T, u, u2, uv, ur)]
        call()
        assert read == [x._version for x in (draft, target, T, u, u2, uv, ur)]
    # what was made by the call itself says so too
    assert all(x._version > 0 for x in (*e, *s, buf, nbytes, *w))
    assert ctx.status()[0] == 0


def test_a_backward_pass_over_what_was_overwritten_is_refused(ctx):
    x, T, _ = _rows()
    q = ctx.compress(_rows(seed=5)[0], T, K, 1.0, K)
    leaf = x.clone().requires_grad_(True)
    # the gradient in place of logits that a loss has saved
    logits = leaf * 1.0
    loss = ctx.distill_loss(logits, T, *q[:3])
    ctx.distill(logits.detach(), T, *q[:3], out=(torch.empty_like(loss), logits.detach()))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()
    # the teacher's rows, taken for the next batch before the backward pass
    loss = ctx.distill_loss(leaf * 1.0, T, *q[:3])
    ctx.compress(_rows(seed=6)[0], T, K, 1.0, K, out=q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()
    ctx.distill_loss(leaf * 1.0, T, *q[:3]).sum().backward()


def test_tensors_of_inference_mode(ctx):
    with torch.inference_mode():
        x, T, u = _rows()
        want = ctx.sample(x, T, u)
        out = tuple(torch.empty_like(t) for t in want)
    ctx.sample(x, T, u, out=out)            # (outside of it such tensors have no version to raise)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    x, T, u = _rows()
    with torch.inference_mode():
        ctx.sample(x, T, u, out=out)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
