"""The norm of many gradients and their clipping against double precision.  fp32 squares are summed over at most 64 entries of a thread in
fp32 (its terms are positive: 64 roundings and one of the square, 65 * 2^-24 of the sum at most, half of that of the norm), the rest in double precision, and the
norm is rounded once: 34 * 2^-24.  A scaled entry is a product with a scale rounded to fp32, rounded itself, and to the type: 2 * 2^-24 + its half
step, relative; the scale inherits nothing of the norm's error but what is stated."""
import numpy as np
import pytest
import torch

from oracle import rules as oracle

pytestmark = pytest.mark.gpu

NORM = 34 * 2.0 ** -24
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(1, 1, 1000, 1)
    yield c
    c.close()


def _np(t):
    return t.detach().float().cpu().numpy()


def _tensors(shapes, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    types = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.float32, torch.bfloat16]}[dtype]
    return [(scale * torch.randn(s, generator=g, device="cuda")).to(types[i % len(types)]) for i, s in enumerate(shapes)]


def _check(ctx, grads, max_norm, scale_tol=NORM + 2 * 2.0 ** -24, atol=2.0 ** -150):
    norm, scale, want = oracle.clip([_np(g) for g in grads], max_norm)
    np.testing.assert_allclose(float(ctx.grad_norm(grads)), norm, rtol=NORM)
    out = [torch.empty_like(g) for g in grads]
    got = ctx.clip_grad(grads, max_norm, out=out)
    np.testing.assert_allclose(float(got), norm, rtol=NORM)
    for o, w, g in zip(out, want, grads):
        np.testing.assert_allclose(_np(o), w, rtol=STEP[g.dtype] + scale_tol, atol=atol)
        if scale == 1.0:
            assert torch.equal(o, g)
    place = [g.clone() for g in grads]
    again = ctx.clip_grad(place, max_norm)
    assert torch.equal(got, again) and all(torch.equal(a, b) for a, b in zip(place, out))
    assert ctx.status()[0] == 0
    return out


SHAPES = [[(1,)], [(3,), (5, 7)], [(0,), (4,), (2, 0)], [(1000,)], [(513, 129), (17,), (2048, 64)], [(65536,), (65537,), (65535,)],
          [(3, 5)] * 70, [(11,)] * 1500, [(1 << 20,), (1,), (333, 777)]]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_norm_and_clipping(ctx, shapes, dtype):
    grads = _tensors(shapes, dtype, len(shapes))
    norm = oracle.clip([_np(g) for g in grads], 1.0)[0]
    for factor in (0.3, 0.999, 1.001, 5.0):
        _check(ctx, grads, float(np.float32(factor * norm)) if norm else 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("front", range(8))
def test_gradients_at_any_offset(ctx, dtype, front):
    # views into a flat buffer, with neighbours that must not move
    flat = torch.randn(40000, device="cuda").to(dtype)
    grads = [flat[front:front + 9001], flat[10000 + front:10000 + front + 3], flat[20000:20000 + front + 8200]]
    before = flat.clone()
    out = _check(ctx, [g for g in grads], 1.0)
    ctx.clip_grad(grads, 1.0)
    touched = torch.zeros(40000, dtype=torch.bool, device="cuda")
    for a, b in ((front, 9001), (10000 + front, 3), (20000, front + 8200)):
        touched[a:a + b] = True
    assert torch.equal(flat[~touched], before[~touched]) and all(torch.equal(g, o) for g, o in zip(grads, out))
    # results at another offset
    other = torch.zeros(40000, device="cuda").to(dtype)
    to = [other[front + 1:front + 1 + 9001], other[10001 + front:10001 + front + 3], other[20003:20003 + front + 8200]]
    flat.copy_(before)
    ctx.clip_grad(grads, 1.0, out=to)
    assert all(torch.equal(a, b) for a, b in zip(to, out)) and torch.equal(flat, before)


def test_a_tensor_of_more_than_2_to_the_31_entries(ctx):
    n = (1 << 31) + 77
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[n - 1], g[1 << 31] = 3.0, 4.0, 12.0
    assert float(ctx.grad_norm([g])) == 13.0
    ctx.clip_grad([g], 6.5)
    assert [float(g[0]), float(g[n - 1]), float(g[1 << 31])] == [1.5, 2.0, 6.0] and int((g != 0).sum()) == 3


def test_a_limit_of_zero_and_one_without_end(ctx):
    g = torch.randn(3000, device="cuda")
    before = g.clone()
    ctx.clip_grad([g], float("inf"))
    assert torch.equal(g, before)
    ctx.clip_grad([g], 0.0)
    assert bool((g == 0).all())
    ctx.clip_grad([g], 0.0)                     # (a norm of zero is not above it)
    assert bool((g == 0).all())


def test_dense_in_any_order(ctx):
    a = torch.randn((300, 500), device="cuda")
    _check(ctx, [a.t(), a.clone().view(10, 30, 500).permute(2, 0, 1)], 3.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-22, 1e18, 1e30, 3e37])
def test_no_gradient_is_too_large_or_too_small(ctx, dtype, size):
    # (entries below fp32's normal range are rounded to its steps of 2^-149, or the type's: absolute)
    grads = [torch.randn(5000, device="cuda").to(dtype) * size, torch.zeros(300000, device="cuda").to(dtype), torch.full((1,), size, device="cuda").to(dtype)]
    norm = oracle.clip([_np(g) for g in grads], 1.0)[0]
    for factor in (0.25, 2.0):
        if factor * norm < 3e38:
            _check(ctx, grads, float(np.float32(factor * norm)), atol=2.0 ** (-149 if dtype == torch.float32 else -133))
    # far below: a scale that is no normal number in fp32
    out = [torch.empty_like(g) for g in grads]
    ctx.clip_grad(grads, 1e-8, out=out)
    scale = min(1.0, float(np.float32(1e-8)) / norm)
    for o, g in zip(out, grads):
        np.testing.assert_allclose(_np(o), _np(g).astype(np.float64) * scale, rtol=STEP[dtype] + NORM + 2 * 2.0 ** -24,
                                   atol=2.0 ** (-149 if dtype == torch.float32 else -133))


def test_a_norm_that_is_not_finite_leaves_the_gradients(ctx):
    for bad in (float("inf"), float("nan")):
        grads = [torch.randn(3000, device="cuda"), torch.randn(100, device="cuda").to(torch.bfloat16)]
        grads[0][1234] = bad
        before = [g.clone() for g in grads]
        norm = float(ctx.clip_grad(grads, 0.5))
        assert norm == float("inf") if bad == float("inf") else norm != norm
        assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(grads, before))


def test_a_norm_of_the_caller(ctx):
    # gradients sharded over ranks: the norm of all of them from each rank's own
    shards = [_tensors([(3000,), (17, 5)], "mixed", s) for s in (1, 2)]
    norms = torch.stack([ctx.grad_norm(s) for s in shards]).double()
    norm = norms.square().sum().sqrt().float().view(1)
    whole = [torch.empty_like(g) for s in shards for g in s]
    ctx.clip_grad([g for s in shards for g in s], 5.0, out=whole)
    for k, s in enumerate(shards):
        assert ctx.clip_grad(s, 5.0, norm=norm) is norm
        for g, w in zip(s, whole[2 * k:2 * k + 2]):
            # (two norms of one value, each NORM off at most, and one rounding of each scale and product)
            np.testing.assert_allclose(_np(g), _np(w), rtol=2 * STEP[g.dtype] + 2 * NORM + 4 * 2.0 ** -24)


def test_results_do_not_depend_on_anything_else(ctx):
    grads = _tensors([(1 << 20,), (999, 77), (1 << 19,)], "mixed", 3)
    want = [ctx.grad_norm(grads) for _ in range(5)]
    side, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got += [ctx.grad_norm(grads) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[0]) for x in want + got)


def test_captured_and_replayed(ctx):
    grads = _tensors([(70000,), (333, 7)], "mixed", 4)
    first = [g.clone() for g in grads]
    ctx.clip_grad(grads, 1.0)
    graphs = []
    for limit in (1.0, 0.5):                # two graphs: each has a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = ctx.clip_grad(grads, limit)
        graphs.append((graph, norm, limit))
    for graph, norm, limit in graphs:
        for g, f in zip(grads, first):
            g.copy_(3 * f)
        want = [torch.empty_like(g) for g in grads]
        want_norm = ctx.clip_grad(grads, limit, out=want)
        graph.replay()
        assert torch.equal(norm, want_norm) and all(torch.equal(a, b) for a, b in zip(grads, want))


def test_versions_and_missing_gradients(ctx):
    grads = _tensors([(10,), (20,)], "f32", 5)
    before = [g._version for g in grads]
    norm = ctx.clip_grad([grads[0], None, grads[1]], 1e-3)
    assert all(g._version > v for g, v in zip(grads, before)) and norm._version > 0
    before = [g._version for g in grads]
    ctx.grad_norm([None, *grads])
    ctx.clip_grad(grads, 1.0, out=[torch.empty_like(g) for g in grads])
    assert [g._version for g in grads] == before
    assert float(ctx.grad_norm([])) == 0.0 and float(ctx.clip_grad([None], 1.0)) == 0.0


def test_refusals(ctx):
    import paper_2603_19133_b200 as ps
    g = torch.randn(100, device="cuda")
    for call in [lambda: ctx.grad_norm([g.half()]), lambda: ctx.grad_norm([g.cpu()]), lambda: ctx.grad_norm([g[::2]]), lambda: ctx.grad_norm([3]),
                 lambda: ctx.grad_norm(5), lambda: ctx.clip_grad([g], -1.0), lambda: ctx.clip_grad([g], float("nan")),
                 lambda: ctx.clip_grad([g, g], 1.0), lambda: ctx.clip_grad([g[:60], g[50:]], 1.0),
                 lambda: ctx.clip_grad([g], 1.0, out=[g.double()]), lambda: ctx.clip_grad([g], 1.0, out=[]), lambda: ctx.clip_grad([g], 1.0, out=[g[:50]]),
                 lambda: ctx.clip_grad([g[:50]], 1.0, out=[g[1:51]]), lambda: ctx.clip_grad([g[:50], g[50:]], 1.0, out=[g[50:], g[:50]]),
                 lambda: ctx.clip_grad([g], 1.0, norm=torch.ones(2, device="cuda"))]:
        before = g.clone()
        with pytest.raises((ValueError, TypeError, ps.PicospecError)):
            call()
        assert torch.equal(g, before)
    # parameters instead of their gradients
    w = torch.nn.Parameter(g.clone())
    for call in (lambda: ctx.clip_grad([w], 1.0), lambda: ctx.clip_grad([g], 1.0, out=[w])):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
    assert torch.equal(w.detach(), g)
    ctx.grad_norm([w])
    with torch.no_grad():
        ctx.clip_grad([w], 1.0)
    # read twice is no overlap
    np.testing.assert_allclose(float(ctx.grad_norm([g, g])), 2 ** 0.5 * float(ctx.grad_norm([g])), rtol=2 * NORM)
    ctx.clip_grad([g, g], 1.0, out=[torch.empty_like(g), torch.empty_like(g)])
