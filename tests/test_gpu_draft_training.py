"""The calls on dense rows together with the sparse rows they stand beside: a teacher's rows are compressed and sent, a student is
trained on them with and without autograd, and tokens are drawn from both."""
import numpy as np
import pytest
import torch

from oracle import rows

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_teacher_rows_over_the_wire_train_a_student(dtype):
    import paper_2603_19133_b200 as ps
    B, R, V, K = 3, 4, 9001, 32
    g = torch.Generator(device="cuda").manual_seed(2)
    teacher = (torch.randn((B, R, V), generator=g, device="cuda") * 2.5).to(dtype)
    student = (teacher.float() * 0.5 + torch.randn((B, R, V), generator=g, device="cuda")).to(dtype)
    T = torch.tensor([0.7, 1.0, 1.3], device="cuda")
    ctx = ps.Context(B, R, V, K)
    try:
        # a token drawn from the teacher's dense rows lies in the sparse rows that keep the same entries
        u = torch.rand((B, R, 2), generator=g, device="cuda")
        k = torch.full((B,), K, dtype=torch.int32, device="cuda")
        token, prob, _, count = ctx.sample(teacher, T, u, k)
        t_idx, t_prob, t_count, _ = ctx.compress(teacher, T, K, 1.0, K)
        assert torch.equal(count, t_count) and bool((t_idx == token[..., None]).any(-1).all())
        # over the wire, as the verifier sends them
        buf, nbytes = ctx.wire_pack(t_idx, t_prob, t_count)
        i2, p2, c2 = ctx.wire_unpack(buf, int(nbytes.item()), B * R, K)
        t_idx, t_prob, t_count = i2.view(B, R, K), p2.view(B, R, K), c2.view(B, R)
        # loss and gradient, by hand and by autograd
        weight = torch.full((B, R), 1.0 / (B * R), device="cuda")
        loss, grad = ctx.distill(student, T, t_idx, t_prob, t_count, weight=weight)
        want_loss, want_grad, _ = rows.distill(_np(student), _np(T), _np(t_idx), _np(t_prob), _np(t_count), _np(weight))
        # (renormalised rows sum to one: 6.6e-6 of the normaliser's logarithm, one rounding)
        np.testing.assert_allclose(_np(loss), want_loss, rtol=2.0 ** -24, atol=6.6e-6)
        # (the normaliser twice at most, against the largest gradient; the gradient's own rounding)
        np.testing.assert_allclose(_np(grad), want_grad, rtol=2.0 ** -8 if dtype == torch.bfloat16 else 3e-5, atol=1.4e-5 * np.abs(want_grad).max())
        leaf = student.clone().requires_grad_(True)
        ctx.distill_loss(leaf, T, t_idx, t_prob, t_count).mean().backward()
        # (the mean's backward pass forms 1 / 12 itself: one step of the type at most)
        torch.testing.assert_close(leaf.grad, grad, rtol=2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -22, atol=0)
        # the raw rows of target_topk, with the rest of the mass
        raw_idx, raw_prob, raw_count = ctx.target_topk(teacher, T, torch.zeros(B, dtype=torch.int32, device="cuda"), K)
        loss, grad = ctx.distill(student[:, :1], T, raw_idx[:, None].contiguous(), raw_prob[:, None].contiguous(),
                                 raw_count[:, None].contiguous(), tail=True)
        want_loss, want_grad, _ = rows.distill(_np(student[:, :1]), _np(T), _np(raw_idx[:, None]), _np(raw_prob[:, None]),
                                               _np(raw_count[:, None]), None, True)
        np.testing.assert_allclose(_np(loss), want_loss, rtol=2.0 ** -24, atol=3 * 6.6e-6)
        # a padded row is left alone, an invalid one (count -1, as compress marks it) is reported
        t_count[0, 0], t_count[1, 1] = 0, -1
        loss, grad = ctx.distill(student, T, t_idx, t_prob, t_count)
        assert float(loss[0, 0]) == 0 and bool((grad[0, 0] == 0).all()) and bool(loss[1, 1].isnan()) and bool(grad[1, 1].isnan().all())
        assert ctx.status(clear=True)[0] == 4
        # the student's own draw, on a stream of its own, from logits made there
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            mine = ctx.sample(student, T, u, k)
        torch.cuda.current_stream().wait_stream(side)
        want = rows.sample(_np(student), _np(T), _np(u), _np(k))
        assert np.array_equal(_np(mine[0]), want[0]) and ctx.status()[0] == 0
    finally:
        ctx.close()


def test_a_step_in_one_graph():
    # sampling, compression, verification and the training step captured together and replayed on new data
    import paper_2603_19133_b200 as ps
    B, G, V, K = 4, 3, 20000, 24
    g = torch.Generator(device="cuda").manual_seed(3)
    target = torch.randn((B, G + 1, V), generator=g, device="cuda") * 2
    draft = torch.randn((B, G, V), generator=g, device="cuda") * 2
    T = torch.ones(B, device="cuda")
    u = torch.rand((B, G + 1, 2), generator=g, device="cuda")
    p = torch.full((B,), 0.9, device="cuda")
    ctx = ps.Context(B, G, V, K)

    def step():
        q_idx, q_prob, q_count, tok = ctx.compress(draft, T, K, 1.0, K, u[:, :G, 0].contiguous())
        out = ctx.verify(target, T, tok, q_idx, q_prob, q_count, u[:, :G, 1].contiguous(), u[:, G].contiguous())
        first = ctx.sample(target, T, u, None, p)
        t_idx, t_prob, t_count, _ = ctx.compress(target[:, :G].contiguous(), T, K, 1.0, K)
        return (out["token"], *first, *ctx.distill(draft, T, t_idx, t_prob, t_count))

    try:
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step()
        for seed in (5, 6):
            g.manual_seed(seed)
            target.copy_(torch.randn(target.shape, generator=g, device="cuda"))
            draft.copy_(torch.randn(draft.shape, generator=g, device="cuda"))
            u.copy_(torch.rand(u.shape, generator=g, device="cuda"))
            graph.replay()
            replayed = [x.clone() for x in captured]
            assert all(torch.equal(a, b) for a, b in zip(replayed, step()))
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_first_calls_of_a_context_inside_a_capture():
    # more rows than clusters run at a time: what the launch asks the device first must not disturb the capture
    import paper_2603_19133_b200 as ps
    B, V, K = 300, 30001, 8
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = torch.randn((B, 1, V), generator=g, device="cuda")
    T, u = torch.ones(B, device="cuda"), torch.rand((B, 1, 2), generator=g, device="cuda")
    t_idx = torch.rand((B, 1, V), generator=g, device="cuda").topk(K, -1).indices.to(torch.int32).contiguous()
    t_prob = torch.full((B, 1, K), 1.0 / K, device="cuda")
    count = torch.full((B, 1), K, dtype=torch.int32, device="cuda")
    ctx = ps.Context(1, 1, V, K)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            drawn = ctx.sample(logits, T, u)
            loss, grad = ctx.distill(logits, T, t_idx, t_prob, count)
        graph.replay()
        assert torch.equal(drawn[0], ctx.sample(logits, T, u)[0])
        again = ctx.distill(logits, T, t_idx, t_prob, count)
        assert torch.equal(loss, again[0]) and torch.equal(grad, again[1])
        # forward and backward of the loss with autograd, captured together
        leaf = logits.clone().requires_grad_(True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            by_autograd, = torch.autograd.grad(ctx.distill_loss(leaf, T, t_idx, t_prob, count).sum(), leaf)
        graph.replay()
        assert torch.equal(by_autograd, grad) and ctx.status()[0] == 0
    finally:
        ctx.close()


def test_both_kernels_are_bracketed_when_profiling():
    import paper_2603_19133_b200 as ps
    V, K = 5000, 4
    logits, T = torch.zeros((2, 1, V), device="cuda"), torch.ones(2, device="cuda")
    t_idx = torch.arange(K, dtype=torch.int32, device="cuda").expand(2, 1, K).contiguous()
    t_prob, count = torch.full((2, 1, K), 0.25, device="cuda"), torch.full((2, 1), K, dtype=torch.int32, device="cuda")
    ctx = ps.Context(1, 1, V, K)
    try:
        ctx.profile_enable(1)
        for _ in range(3):
            ctx.sample(logits, T, torch.zeros((2, 1, 2), device="cuda"))
            ctx.distill(logits, T, t_idx, t_prob, count)
        for kind in (7, 8):
            ms = ctx.profile_samples(kind)
            assert len(ms) == 3 and all(x > 0 for x in ms)
        ctx.profile_enable(0)
    finally:
        ctx.close()
