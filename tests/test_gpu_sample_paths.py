"""The ways a row can take through the sampling kernel, with clusters of several CTAs and more rows than run at a time: CTAs end at
different times and others take their places on the SM."""
import pytest
import torch

from test_gpu_sample import _check, _stored, _uniforms, _zipf, ps  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,V", [("bf16", 140001), ("f32", 70001)])
def test_min_p_alone_in_many_rows(ps, dtype, V):
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = _stored(_zipf(160, 2, V, g), dtype)
    T = 0.4 + torch.rand((160,), generator=g, device="cuda")
    _check(ps, logits, T, _uniforms(160, 2, g), None, None, 1e-3 + torch.rand((160,), generator=g, device="cuda") ** 3)


def test_entries_of_a_bin_put_in_order_in_many_rows(ps):
    g = torch.Generator(device="cuda").manual_seed(43)
    V = 70001
    logits = _stored(_zipf(160, 2, V, g), "f32")
    T = 0.4 + torch.rand((160,), generator=g, device="cuda")
    k = torch.randint(1, 1200, (160,), generator=g, device="cuda", dtype=torch.int32)
    p = 0.3 + 0.69 * torch.rand((160,), generator=g, device="cuda")
    _check(ps, logits, T, _uniforms(160, 2, g), k)
    _check(ps, logits, T, _uniforms(160, 2, g), None, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_draws_on_borders_of_chunks_in_many_rows(ps, dtype):
    # no limits; 64 chunks of the same mass: a uniform of j / 64 lies on a border, so every row takes its exact sums
    g = torch.Generator(device="cuda").manual_seed(47)
    V, n = 65536, 400
    logits = _stored(torch.full((1, 1, 1), 0.5, device="cuda").expand(n, 1, V), dtype)
    u = _uniforms(n, 1, g)
    u[:, 0, 0] = torch.randint(0, 64, (n,), generator=g, device="cuda") / 64.0
    got, slow = _check(ps, logits, torch.ones(n, device="cuda"), u)
    assert slow == int((u[:, 0, 0] > 0).sum())
    assert torch.equal(got[0][:, 0] // 1024, (u[:, 0, 0] * 64).to(torch.int32))


@pytest.mark.parametrize("limits", [False, True])
@pytest.mark.parametrize("dtype,V", [("bf16", 90001), ("f32", 60001)])
def test_late_waits_mark_whole_rows(ps, dtype, V, limits):
    # with a limit of zero a wait that is not complete yet gives its row up: in every CTA of the cluster and in every output, or not at all
    g = torch.Generator(device="cuda").manual_seed(53)
    n = 600
    base = _stored(_zipf(1, 1, V, g).expand(n, 1, V), dtype)
    T, u = 0.5 + torch.rand((n,), generator=g, device="cuda"), _uniforms(n, 1, g)
    k = torch.randint(0, 300, (n,), generator=g, device="cuda", dtype=torch.int32) if limits else None
    ctx = ps.Context(1, 1, V, 1)
    try:
        want = ctx.sample(base, T, u, k)
        assert ctx.status()[0] == 0
        ctx.wait_limit(0)
        for _ in range(4):
            token, prob, logprob, count = ctx.sample(base, T, u, k)
            assert ctx.status(clear=True)[0] == 8
            late = token == -1
            assert bool(late.any()) and torch.equal(late, count == -1) and torch.equal(late, prob == -1) and torch.equal(late, logprob.isnan())
            for a, b in zip((token, prob, logprob, count), want):
                assert torch.equal(a[~late], b[~late])
        ctx.wait_limit(2_000_000_000)
        assert all(torch.equal(a, b) for a, b in zip(ctx.sample(base, T, u, k), want)) and ctx.status()[0] == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("limits", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_of_nothing_but_nan_are_bad_logits(ps, dtype, limits):
    # (they have no maximum; a wait that ran out is another matter, and would have later calls on the context marked too)
    g = torch.Generator(device="cuda").manual_seed(59)
    V = 20000
    logits = _stored(_zipf(4, 1, V, g), dtype)
    logits[0] = float("nan")
    logits[1, 0, 4096:5120] = float("nan")
    logits[2, 0, 19456:] = float("nan")
    k = torch.full((4,), 40, dtype=torch.int32, device="cuda") if limits else None
    _check(ps, logits, torch.ones(4, device="cuda"), _uniforms(4, 1, g), k, status=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5000, 60001])
def test_fewer_finite_entries_than_top_k(ps, dtype, V):
    # a grammar's mask: the sample of one entry in 32 finds next to nothing, and the range that it leaves is empty
    g = torch.Generator(device="cuda").manual_seed(61)
    n = 96
    x = torch.full((n, 1, V), -float("inf"), device="cuda")
    finite = torch.randint(1, 180, (n,), generator=g, device="cuda")
    for b in range(n):
        at = torch.randperm(V, generator=g, device="cuda")[:int(finite[b])]
        x[b, 0, at] = 2 * torch.randn(at.numel(), generator=g, device="cuda")
    logits, u = _stored(x, dtype), _uniforms(n, 1, g)
    T = 0.4 + torch.rand((n,), generator=g, device="cuda")
    k = torch.randint(180, min(V, 3000), (n,), generator=g, device="cuda", dtype=torch.int32)
    p = 0.99 + 0.02 * torch.rand((n,), generator=g, device="cuda")
    tiny = torch.full((n,), 1e-10, device="cuda")
    got, _ = _check(ps, logits, T, u, k)
    assert torch.equal(got[3][:, 0], finite.to(torch.int32))
    _check(ps, logits, T, u, k, p)
    _check(ps, logits, T, u, k, None, tiny)
    _check(ps, logits, T, u, k, p, tiny)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e30, 5e36, 1e38, 3.4e38])
def test_masked_entries_weigh_nothing_at_any_temperature(ps, dtype, T):
    # so large a temperature that the lowest finite logit weighs about as much as the largest: -inf still has no weight
    g = torch.Generator(device="cuda").manual_seed(67)
    n, V = 40, 16384            # (rows on 16 bytes, whole chunks)
    x = torch.randn((n, 1, V), generator=g, device="cuda")
    x[:20] *= 1e37
    x[torch.rand((n, 1, V), generator=g, device="cuda") < 0.6] = -float("inf")
    logits, u = _stored(x, dtype), _uniforms(n, 1, g)
    temperature = torch.full((n,), T, device="cuda")
    p = 0.05 + 0.9 * torch.rand((n,), generator=g, device="cuda")
    k = torch.randint(1, 9000, (n,), generator=g, device="cuda", dtype=torch.int32)
    _check(ps, logits, temperature, u)
    _check(ps, logits, temperature, u, None, p)
    _check(ps, logits, temperature, u, k)
    _check(ps, logits, temperature, u, k, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_min_p_far_from_its_logit(ps, dtype):
    # the bound on the logit lies at the lowest values that there are, or where weights of many of them round to the same
    g = torch.Generator(device="cuda").manual_seed(71)
    n, V = 48, 6000
    u = _uniforms(n, 1, g)
    lowest = torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min
    x = torch.randn((n, 1, V), generator=g, device="cuda")
    x[..., : V // 2] = lowest * (0.9 + 0.1 * torch.rand((n, 1, V // 2), generator=g, device="cuda"))
    T = torch.full((n,), 1e38, device="cuda")
    m = torch.exp(-3.403 * (0.96 + 0.05 * torch.rand((n,), generator=g, device="cuda")))      # T ln m from 0.96 of the lowest to beyond it
    _check(ps, _stored(x, dtype), T, u, None, None, m)
    _check(ps, _stored(x, dtype), T, u, torch.full((n,), 4000, dtype=torch.int32, device="cuda"), None, m)
    _check(ps, _stored(x, dtype), torch.full((n,), 3.4e38, device="cuda"), u, None, None, 0.3 + 0.7 * m)
    # min_p of 1, and next to it, where all weights round to 1 in double precision: the largest logit alone, and every one
    x = torch.randn((n, 1, V), generator=g, device="cuda") * 5
    one = torch.ones(n, device="cuda")
    for t in (1e10, 1e18, 1e30):
        got, _ = _check(ps, _stored(x, dtype), t * one, u, None, None, one)
        logits = _stored(x, dtype)
        assert torch.equal(got[3], (logits == logits.amax(-1, keepdim=True)).sum(-1, dtype=torch.int32))
        _check(ps, _stored(x, dtype), t * one, u, None, None, one - 2.0 ** -24)
    # a bound next to zero, where the values lie close
    x[..., ::3] *= 10.0 ** -(30 * torch.rand((n, 1, V // 3), generator=g, device="cuda"))
    x = x.clamp(max=1.0)
    for s in (1 - 1e-6, 1.0, 1 + 1e-6):
        _check(ps, _stored(x, dtype), one, u, None, None, torch.exp(-one * s))
