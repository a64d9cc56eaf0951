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
