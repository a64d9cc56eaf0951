"""Norms and clipped gradients depend on the gradients alone: not on where in memory they lie, and not on whether the norm is taken within the
call or handed to it.  Everything here is equal bit by bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(1, 1, 1000, 1)
    yield c
    c.close()


def _bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def _views(dtype, front, seed, sizes=(9001, 3, 8200, 16385)):
    """Neighbouring views that start `front` elements behind a 16-byte boundary."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat, at, out = torch.randn(sum(sizes) + 64 * len(sizes), generator=g, device="cuda").to(dtype), 0, []
    for n in sizes:
        out.append(flat[at + front:at + front + n])
        at += (n + front + 15) // 8 * 8
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("front", range(8))
def test_where_gradients_lie_makes_no_difference(ctx, dtype, front):
    for seed in range(40):
        views = _views(dtype, front, seed)
        aligned = [v.clone() for v in views]
        assert torch.equal(ctx.grad_norm(views), ctx.grad_norm(aligned)), seed
        out = [torch.empty_like(v) for v in aligned]
        assert torch.equal(ctx.clip_grad(views, 1.0, out=out), ctx.clip_grad(aligned, 1.0)), seed
        assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(out, aligned)), seed
    assert ctx.status()[0] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sizes_around_granules_and_tiles_at_every_offset(ctx, dtype):
    # the sum itself, of small whole numbers: exact in fp32 whatever the order, so an entry that is missed or taken twice shows
    n = 8 if dtype == torch.bfloat16 else 4
    sizes = [*range(0, 2 * n + 2), 256 * n - 1, 256 * n, 256 * n + 1, 2048 * n - 1, 2048 * n, 2048 * n + 1, 2049 * n + 1, 4096 * n + 3]
    for front in range(8):
        for size in sizes:
            flat = torch.full((size + 24,), 64.0, device="cuda").to(dtype)          # (what must not be counted)
            view = flat[front:front + size]
            view.copy_(torch.arange(size, device="cuda") % 2 + 1)
            want = torch.tensor([float((view.double() ** 2).sum())], device="cuda", dtype=torch.float64).sqrt().float()
            assert torch.equal(ctx.grad_norm([view]), want), (front, size)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_norm_taken_before_gives_what_one_taken_within_gives(ctx, dtype):
    for seed in range(60):
        grads = _views(dtype, 0, seed, sizes=(9001, 3, 70001))
        for limit in (1.0, 0.37, 250.0):
            out, own = ([torch.empty_like(g) for g in grads] for _ in range(2))
            norm = ctx.grad_norm(grads)
            ctx.clip_grad(grads, limit, norm=norm, out=out)
            assert torch.equal(ctx.clip_grad(grads, limit, out=own), norm)
            assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(out, own)), (seed, limit)
    # at the norm itself nothing is clipped, a step below all is
    before = [g.clone() for g in grads]
    ctx.clip_grad(grads, float(norm))
    assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(grads, before))
    assert ctx.status()[0] == 0


def test_a_norm_beyond_fp32(ctx):
    # 2^127 four times 64: a norm of 2^131 is returned as inf; the gradients are scaled all the same, unless that inf is handed in
    grads = [torch.full((256,), 2.0 ** 127, device="cuda")]
    out = [torch.empty_like(grads[0])]
    norm = ctx.clip_grad(grads, 16.0, out=out)
    assert float(norm) == float("inf") and bool((out[0] == 1.0).all()) and float(ctx.grad_norm(grads)) == float("inf")
    ctx.clip_grad(grads, 16.0, norm=norm, out=out)
    assert torch.equal(out[0], grads[0])
    # below fp32's normal range: 2^-140 four times is a norm of 2^-139, of 2^-149 a norm of 2^-148
    for e in (140, 149):
        tiny = [torch.full((4,), 2.0 ** -e, device="cuda")]
        assert float(ctx.grad_norm(tiny)) == 2.0 ** (1 - e)
        ctx.clip_grad(tiny, 2.0 ** -130)
        assert bool((tiny[0] == 2.0 ** -e).all())
