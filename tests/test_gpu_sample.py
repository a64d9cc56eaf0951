"""Sampling from dense rows on the GPU against the double-precision statement (oracle/rows.py).  Tokens and counts are
exact.  A truncated row's probability is a quotient of double-precision sums, rounded once: 2^-24 (and 1e-12 for the order of
the sums).  Z, and the mass of a row without truncation, is accumulated in fp32: 3e-6 (GUARD_Z)."""
import numpy as np
import pytest
import torch

from oracle import rows

pytestmark = pytest.mark.gpu

GUARD_Z = 3e-6


@pytest.fixture(scope="module")
def ps():
    import paper_2603_19133_b200 as ps
    ps.lib()
    return ps


def _np(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _stored(values, dtype, pad=0, front=0):
    """In rows of V + pad elements (NaN between them) that start `front` elements late."""
    B, R, V = values.shape
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((B * R * (V + pad) + front,), float("nan"), dtype=td, device="cuda")
    logits = buf[front:].view(B, R, V + pad)[..., :V]
    logits.copy_(values)
    return logits


def _zipf(B, R, V, g, offset=0.0):
    base = torch.rand((B, R, V), generator=g, device="cuda").mul_(V - 1).add_(1).log_().mul_(-1.1)
    return base + 1.5 * torch.randn((B, R, V), generator=g, device="cuda") + offset


def _uniforms(B, R, g):
    return torch.rand((B, R, 2), generator=g, device="cuda").clamp_(max=1 - 2.0 ** -24)


def _check(ps, logits, T, u, k=None, p=None, m=None, status=0, ctx=None):
    own = ctx is None
    ctx = ctx or ps.Context(1, 1, logits.shape[-1], 1)
    try:
        got = ctx.sample(logits, T, u, k, p, m)
        st, slow = ctx.status(clear=True)
    finally:
        if own:
            ctx.close()
    want = rows.sample(_np(logits), _np(T), _np(u), *[None if x is None else _np(x) for x in (k, p, m)])
    assert st == status
    assert np.array_equal(_np(got[3]), want[3]), ("count", _np(got[3]), want[3])
    assert np.array_equal(_np(got[0]), want[0]), ("token", _np(got[0]), want[0])
    np.testing.assert_allclose(_np(got[1]), want[1], rtol=2.0 ** -24 + GUARD_Z, atol=2.0 ** -149)
    np.testing.assert_allclose(_np(got[2]), want[2], rtol=2.0 ** -24, atol=GUARD_Z)
    limited = np.zeros(want[0].shape, bool)
    V = logits.shape[-1]
    for x, on in ((k, lambda x: (x > 0) & (x < V)), (p, lambda x: x < 1), (m, lambda x: x > 0)):
        if x is not None:
            limited |= on(_np(x))[:, None]
    np.testing.assert_allclose(_np(got[1])[limited], want[1][limited], rtol=2.0 ** -24 + 1e-12, atol=2.0 ** -149)
    return got, slow


LAWS = {
    "plain": lambda B, g: (None, None, None),
    "k": lambda B, g: (torch.randint(1, 1200, (B,), generator=g, device="cuda", dtype=torch.int32), None, None),
    "p": lambda B, g: (None, 0.3 + 0.69 * torch.rand((B,), generator=g, device="cuda"), None),
    "m": lambda B, g: (None, None, torch.rand((B,), generator=g, device="cuda") ** 3),
    "kpm": lambda B, g: (torch.randint(0, 300, (B,), generator=g, device="cuda", dtype=torch.int32),
                         0.5 + 0.6 * torch.rand((B,), generator=g, device="cuda"),
                         0.02 * torch.rand((B,), generator=g, device="cuda")),
}


@pytest.mark.parametrize("law", list(LAWS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,R,V,pad,front", [
    (3, 1, 1, 0, 0),
    (2, 3, 2, 0, 0),
    (4, 2, 100, 3, 1),
    (3, 2, 1024, 0, 0),
    (3, 2, 1025, 0, 0),            # a chunk and one entry; rows at any offset
    (2, 2, 8193, 8, 0),
    (6, 2, 32000, 0, 0),
    (5, 2, 50381, 0, 3),
    (4, 1, 128256, 0, 0),
    (2, 1, 262144, 5, 0),
])
def test_every_law(ps, B, R, V, pad, front, dtype, law):
    g = torch.Generator(device="cuda").manual_seed(V + len(law))
    T = 0.4 + torch.rand((B,), generator=g, device="cuda")
    logits = _stored(_zipf(B, R, V, g), dtype, pad, front)
    _check(ps, logits, T, _uniforms(B, R, g), *LAWS[law](B, g))


@pytest.mark.parametrize("dtype,V", [("bf16", 688120), ("f32", 344056)])
def test_the_longest_rows(ps, dtype, V):
    g = torch.Generator(device="cuda").manual_seed(V)
    T = torch.tensor([0.7, 1.0, 1.3], device="cuda")
    logits = _stored(_zipf(3, 1, V, g), dtype)
    _check(ps, logits, T, _uniforms(3, 1, g), torch.tensor([0, 50, 0], dtype=torch.int32, device="cuda"),
           torch.tensor([1.0, 1.0, 0.9], device="cuda"), None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows_", [40, 149, 400])
def test_many_rows(ps, rows_, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows_)
    T = 0.5 + torch.rand((rows_,), generator=g, device="cuda")
    logits = _stored(_zipf(rows_, 1, 20000, g), dtype)
    k, p, m = LAWS["kpm"](rows_, g)
    got, slow = _check(ps, logits, T, _uniforms(rows_, 1, g), k, p, m)
    assert slow < rows_ // 2


@pytest.mark.parametrize("offset", [20.0, -40.0, 300.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_around_a_common_offset(ps, dtype, offset):
    # bf16: a few hundred values share the row, ties at every cut; across zero the bit patterns lie far apart
    g = torch.Generator(device="cuda").manual_seed(7)
    logits = _stored(_zipf(6, 2, 30000, g, offset), dtype)
    T = torch.full((6,), 0.9, device="cuda")
    for law in ("k", "p", "kpm"):
        _check(ps, logits, T, _uniforms(6, 2, g), *LAWS[law](6, g))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,p,m", [(1, 1.0, 0.0), (2, 1.0, 0.0), (4999, 1.0, 0.0), (5000, 1.0, 0.0), (0, 1e-7, 0.0), (0, 0.5, 0.0),
                                   (0, 0.9999999, 0.0), (0, 1.0, 1.0), (0, 1.0, 0.999), (3000, 0.7, 0.5)])
def test_all_entries_equal(ps, dtype, k, p, m):
    V = 5000
    logits = _stored(torch.full((1, 64, V), 1.375, device="cuda"), dtype)
    g = torch.Generator(device="cuda").manual_seed(k)
    one = torch.ones(1, device="cuda")
    _check(ps, logits, one, _uniforms(1, 64, g), torch.tensor([k], dtype=torch.int32, device="cuda"), one * p, one * m)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_flat_rows_and_wide_rows(ps, dtype):
    # nearly uniform: every cut lies among entries worth less than the error of an fp32 sum, so the exact one decides
    g = torch.Generator(device="cuda").manual_seed(3)
    p = torch.tensor([0.05, 0.5, 0.95, 0.9999, 1.0 - 2.0 ** -24], device="cuda")
    T = torch.full((5,), 1.0, device="cuda")
    flat = _stored(torch.rand((5, 2, 40000), generator=g, device="cuda") * 1e-3, dtype)
    _, slow = _check(ps, flat, T, _uniforms(5, 2, g), None, p)
    assert slow > 0
    k = torch.tensor([1, 3000, 20000, 39999, 40000], dtype=torch.int32, device="cuda")
    _check(ps, flat, T, _uniforms(5, 2, g), k)
    _check(ps, flat, T, _uniforms(5, 2, g), None, None, torch.tensor([0.9991, 0.9995, 0.9999, 1.0, 0.5], device="cuda"))
    # a range of 1e30: nothing but the largest has weight, yet top-k counts
    wide = torch.randn((5, 2, 40000), generator=g, device="cuda")
    wide = _stored(wide.sign() * 10.0 ** (wide.abs() * 10 - 8), dtype)
    _check(ps, wide, T, _uniforms(5, 2, g), k)
    _check(ps, wide, T, _uniforms(5, 2, g), None, p)
    _check(ps, wide, T * 1e-30, _uniforms(5, 2, g), k, p)
    _check(ps, wide, T * 1e30, _uniforms(5, 2, g), k, p)
    # top-p where a few bins are wide: one large entry, all others 60 nats below, spread over thousands of values
    low = torch.rand((5, 2, 40000), generator=g, device="cuda") * 60 + 5
    low[..., 17] = 70.0
    _check(ps, _stored(low, dtype), T * 30, _uniforms(5, 2, g), None, p)
    _check(ps, _stored(low, dtype), T, _uniforms(5, 2, g), None, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_and_bad_data(ps, dtype):
    V = 9000
    g = torch.Generator(device="cuda").manual_seed(11)
    x = _zipf(8, 2, V, g)
    x[0, 0, 1:] = -float("inf")                     # one entry is left
    x[0, 1, ::2] = -float("inf")
    lowest = torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min
    x[1, 0, 100:] = lowest
    x[1, 1, :] = lowest                             # nothing but the lowest value: a uniform row
    logits = _stored(x, dtype, pad=3)
    logits[2, 0, 5] = float("nan")
    logits[2, 1, 8999] = float("inf")
    logits[3, 0, :] = -float("inf")
    logits[3, 1, :] = -float("inf")
    logits[3, 1, 4000] = float("nan")               # a NaN among nothing else
    T = torch.full((8,), 0.8, device="cuda")
    T[4] = 0.0
    k = torch.tensor([50, 200, 50, 50, 50, -1, 50, 50], dtype=torch.int32, device="cuda")
    p = torch.tensor([0.9, 0.9, 0.9, 0.9, 0.9, 0.9, float("nan"), 0.9], device="cuda")
    m = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 1.5], device="cuda")
    u = _uniforms(8, 2, g)
    got, _ = _check(ps, logits, T, u, k, p, m, status=1 | 2 | 4)
    assert _np(got[0])[0, 0] == 0 and list(_np(got[3])[2:, 0]) == [-1] * 6
    _check(ps, logits[:2], T[:2], u[:2])            # masked rows without truncation: the finite entries count
    _check(ps, logits[:2], T[:2], u[:2], torch.tensor([8000, 8999], dtype=torch.int32, device="cuda"))
    _check(ps, logits[:2], T[:2], u[:2], None, p[:2])
    _check(ps, logits[:2], T[:2], u[:2], None, None, m[:2] + 1e-3)


@pytest.mark.parametrize("truncated", [False, True])
def test_uniforms_at_the_ends_and_at_borders(ps, truncated):
    # chunk masses 1 : 1 : 2 exactly, entries of equal weight: u = 1/4, 1/2 lie on a chunk's border, which the strict
    # comparison gives to the next chunk; a step of fp32 below lies in the chunk before
    V = 4096
    x = torch.zeros((1, 1, V), device="cuda")
    us = [0.0, 0.25, 0.25 - 2.0 ** -26, 0.5, 0.5 - 2.0 ** -25, 1 - 2.0 ** -24, 1e-9]
    u = torch.tensor([[a, b] for a in us for b in us], device="cuda")
    n = u.shape[0]
    logits = _stored(x.expand(1, n, V), "f32")
    T = torch.ones(1, device="cuda")
    k = torch.tensor([3000], dtype=torch.int32, device="cuda") if truncated else None
    _check(ps, logits, T, u[None].contiguous(), k)


def test_the_same_as_the_sparse_rows_law(ps):
    # top-k and top-p keep what Context.compress keeps, and prob is its probability
    g = torch.Generator(device="cuda").manual_seed(13)
    logits = _stored(_zipf(8, 3, 32000, g), "bf16")
    T = torch.full((8,), 0.8, device="cuda")
    k, p = torch.full((8,), 64, dtype=torch.int32, device="cuda"), torch.full((8,), 0.9, device="cuda")
    ctx = ps.Context(8, 3, 32000, 64)
    try:
        qi, qp, qc, _ = ctx.compress(logits, T, 64, 0.9, 64)
        token, prob, _, count = ctx.sample(logits, T, _uniforms(8, 3, g), k, p)
        assert torch.equal(count, qc)
        hit = (qi == token[..., None]) & (torch.arange(64, device="cuda") < qc[..., None])
        assert bool((hit.sum(-1) == 1).all())
        torch.testing.assert_close((qp * hit).sum(-1), prob, rtol=1e-5, atol=0)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_outputs_strides_and_refusals(ps):
    g = torch.Generator(device="cuda").manual_seed(17)
    logits = _stored(_zipf(4, 2, 3000, g), "bf16")
    T, u = torch.ones(4, device="cuda"), _uniforms(4, 2, g)
    k, p, m = LAWS["kpm"](4, g)
    ctx = ps.Context(1, 1, 3000, 1)
    try:
        f = ctx.sample
        want = f(logits, T, u, k, p, m)
        token = torch.empty_like(want[0])
        assert f(logits, T, u, k, p, m, out=(token, None, None, None))[0] is token and torch.equal(token, want[0])
        again = f(logits, T, u, k, p, m)
        assert all(torch.equal(a, b) for a, b in zip(want, again))
        assert torch.equal(f(logits[:, 1:2], T, u[:, 1:2].contiguous(), k, p, m)[0], want[0][:, 1:2])     # a view of every other row
        for args in [(logits.half(), T, u), (logits[0], T, u), (logits, T[:1], u), (logits, T, u[..., :1]),
                     (logits, T, u.double()), (logits.cpu(), T, u), (logits, T.cpu(), u), (logits, T, u, k.long()),
                     (logits, T, u, k[:1]), (logits, T, u, None, p.double()), (logits, T, u, None, None, m.cpu()),
                     (logits.transpose(1, 2), T, u), (logits, T, u.transpose(0, 1))]:
            with pytest.raises(ValueError):
                f(*args)
        with pytest.raises(ps.PicospecError) as e:
            f(torch.zeros((4, 2, 3001), device="cuda"), T, u)
        assert e.value.code == -3
        with pytest.raises(ps.PicospecError) as e:
            f(logits, T, u, out=(None, None, None, None))
        assert e.value.code == -1
        big = ps.Context(1, 1, 500000, 1)
        with pytest.raises(ps.PicospecError) as e:
            big.sample(torch.zeros((4, 2, 344057), device="cuda"), T, u)
        assert e.value.code == -3
        big.close()
        empty = f(logits[:0], T[:0], u[:0])
        assert all(x.shape == (0, 2) for x in empty)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_captured_replayed_and_on_other_streams(ps):
    g = torch.Generator(device="cuda").manual_seed(19)
    logits, T, u = _stored(_zipf(60, 1, 40000, g), "bf16"), torch.ones(60, device="cuda"), _uniforms(60, 1, g)
    k, p, m = LAWS["kpm"](60, g)
    ctx = ps.Context(1, 1, 40000, 1)
    try:
        want = ctx.sample(logits, T, u, k, p, m)
        outs = []
        for s in [torch.cuda.Stream() for _ in range(2)]:       # two at once on one context
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs += [ctx.sample(logits, T, u, k, p, m) for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o in outs for a, b in zip(o, want))
        out = tuple(torch.empty_like(x) for x in want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.sample(logits, T, u, k, p, m, out=out)
        for _ in range(3):
            out[0].fill_(-7)
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        u.copy_(_uniforms(60, 1, g))
        graph.replay()
        assert torch.equal(out[0], ctx.sample(logits, T, u, k, p, m)[0])
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_a_wait_that_runs_out_marks_the_rows(ps):
    g = torch.Generator(device="cuda").manual_seed(23)
    logits, T, u = _stored(_zipf(3, 1, 60000, g), "bf16"), torch.ones(3, device="cuda"), _uniforms(3, 1, g)
    ctx = ps.Context(1, 1, 60000, 1)
    try:
        ctx.wait_limit(0)
        got = ctx.sample(logits, T, u)
        status = ctx.status(clear=True)[0]
        assert (status == 8) == bool((got[0] == -1).any())
        ctx.wait_limit(2_000_000_000)
        _check(ps, logits, T, u, ctx=ctx)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zeros_of_either_sign_tie(ps, dtype):
    # -0 and +0 are one value: of those that tie at the cut the lowest indices are kept
    V = 3000
    x = torch.zeros((1, 32, V), device="cuda")
    x[..., 1::2] = -0.0
    x[..., 100:] -= 1.0
    g = torch.Generator(device="cuda").manual_seed(29)
    logits, one = _stored(x, dtype), torch.ones(1, device="cuda")
    for k in (1, 7, 50, 99, 100, 101):
        got, _ = _check(ps, logits, one, _uniforms(1, 32, g), torch.tensor([k], dtype=torch.int32, device="cuda"))
        assert int(got[0].max()) < max(k, 100)
    _check(ps, logits, one, _uniforms(1, 32, g), None, 0.3 * one)
    _check(ps, logits, one, _uniforms(1, 32, g), None, None, one)


def test_rows_without_limits_beside_rows_with_them(ps):
    # limits that are given but off, in the same call as limits that are on; equal to the call that has none
    g = torch.Generator(device="cuda").manual_seed(31)
    logits, T, u = _stored(_zipf(6, 2, 33000, g), "bf16"), torch.ones(6, device="cuda"), _uniforms(6, 2, g)
    k = torch.tensor([0, 33000, 40000, 5, 0, 0], dtype=torch.int32, device="cuda")
    p = torch.tensor([1.0, 1.5, 1.0, 1.0, 0.5, 1.0], device="cuda")
    m = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.0, 0.5], device="cuda")
    got, _ = _check(ps, logits, T, u, k, p, m)
    plain, _ = _check(ps, logits, T, u)
    assert all(torch.equal(a[:3], b[:3]) for a, b in zip(got, plain))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at_samples", [-50.0, 1.5, 60.0])
def test_rows_that_mislead_the_sample(ps, dtype, at_samples):
    # every entry that the kernel's sample of one in 32 looks at lies far from the others: its bracket is wrong and has to be
    # taken back
    V = 20480
    c, lane = np.meshgrid(np.arange(V // 1024), np.arange(32), indexing="ij")
    at = torch.from_numpy((c * 1024 + lane * 32 + ((lane * 7 + c * 11) & 31)).reshape(-1)).cuda()
    g = torch.Generator(device="cuda").manual_seed(37)
    x = torch.randn((6, 2, V), generator=g, device="cuda") * 0.3
    x[..., at] = at_samples + 0.1 * torch.randn((6, 2, at.numel()), generator=g, device="cuda")
    logits, T = _stored(x, dtype), torch.full((6,), 1.0, device="cuda")
    p = torch.tensor([0.3, 0.9, 0.99, 0.999, 0.5, 1.0], device="cuda")
    k = torch.tensor([0, 0, 0, 0, 9000, 15000], dtype=torch.int32, device="cuda")
    _check(ps, logits, T, _uniforms(6, 2, g), k, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("step", [0.5, 0.25, 1e-3])
def test_many_zeros_among_values_of_both_signs(ps, dtype, step):
    # no logit has the bit pattern between those of 0 and of the negative values; cuts at, just above and just below 0
    g = torch.Generator(device="cuda").manual_seed(41)
    V = 19522
    x = torch.round(torch.randn((24, 1, V), generator=g, device="cuda") / step * 0.5) * step
    logits = _stored(x, dtype)
    T = torch.exp(torch.rand((24,), generator=g, device="cuda") * 3 - 1.5)
    above = (logits > 0).sum(-1)[:, 0]
    at = torch.tensor([-1, 0, 1, 2], device="cuda").repeat(6) + torch.cat([above[:12], (logits >= 0).sum(-1)[12:, 0]])
    _check(ps, logits, T, _uniforms(24, 1, g), at.clamp(min=1).to(torch.int32))
    w = torch.exp((logits.double() - logits.double().amax(-1, keepdim=True)) / T[:, None, None])
    share = (w * (logits > 0)).sum(-1) / w.sum(-1), (w * (logits >= 0)).sum(-1) / w.sum(-1)
    for s in (share[0] - 1e-3, share[0] + 1e-3, share[1] - 1e-3, share[1] + 1e-3):
        _check(ps, logits, T, _uniforms(24, 1, g), None, s[:, 0].clamp(1e-3, 1.0).float())
    m = torch.exp(-logits.float().amax(-1)[:, 0] / T)
    for s in (0.999, 1.001):
        _check(ps, logits, T, _uniforms(24, 1, g), None, None, (m * s).clamp(max=1.0))
