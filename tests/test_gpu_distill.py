"""Distillation from a teacher's top entries on the GPU against the double-precision statement (oracle/rows.py).

Tolerances, from the arithmetic of the kernel (before its first run):
  a streaming sum carries 3e-6 (GUARD_Z: ex2, the exponent's rounding, accumulation), at most 13 changes of reference a
  warp and two factors between warps, at 2^-22 each: 6.6e-6 in all = Z.  ln of it carries Z as well.  (ln t in fp32 adds
  2^-22 of sum t |ln t|, under Z by the roundings that never come together.)
  loss      A Z from ln s, r 2 Z from ln R, one rounding to fp32 (2^-24)
  gradient  on the entries: (A + r) s Z, one rounding
            elsewhere: g = ((A + r) R - r) s / R: 2 Z on R (a ratio of sums), and on s / R: Z, 2^-22 (ex2), and per term
            with s / max s = 2^-x: x ln 2 (2^-24 + 2^-24) (scale and exponent) + 2^-24; one rounding of the coefficient
  a rounding to bf16 is 2^-8 relative (2^-134 below the normal range), to fp32 2^-24 (2^-126 where ex2 flushes, times weight / T)
"""
import numpy as np
import pytest
import torch

from oracle import rows

pytestmark = pytest.mark.gpu

Z = 6.6e-6


@pytest.fixture(scope="module")
def ps():
    import paper_2603_19133_b200 as ps
    ps.lib()
    return ps


def _np(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _inputs(B, R, V, K, dtype, seed, pad=0, offset=0.0, total=None, spread=2.0, front=0):
    """Student rows in a buffer of V + pad elements a row (NaN between them) that starts `front` elements late."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((B * R * (V + pad) + front,), float("nan"), dtype=td, device="cuda")
    logits = buf[front:].view(B, R, V + pad)[..., :V]
    logits.copy_(torch.randn((B, R, V), generator=g, device="cuda") * spread + offset)
    idx = torch.rand((B, R, V), generator=g, device="cuda").topk(K, -1).indices.to(torch.int32).contiguous()
    t = torch.rand((B, R, K), generator=g, device="cuda") ** 4
    t = t / t.sum(-1, keepdim=True) * (1.0 if total is None else total)
    count = torch.randint(1, K + 1, (B, R), generator=g, device="cuda", dtype=torch.int32)
    count[0, 0] = K
    weight = torch.rand((B, R), generator=g, device="cuda")
    T = 0.5 + torch.rand((B,), generator=g, device="cuda")
    return logits, T, idx, t, count, weight


def _check(got, logits, T, idx, t, count, weight, tail):
    l, Tn, tn, n = _np(logits), _np(T), _np(t), _np(count)
    w = np.ones(n.shape) if weight is None else _np(weight).astype(np.float64)
    loss, grad, out = rows.distill(l, Tn, _np(idx), tn, n, w, tail)
    valid = np.arange(t.shape[-1]) < n[..., None]
    A = (tn.astype(np.float64) * valid).sum(-1)
    r = np.maximum(0, 1 - A) * (n > 0) if tail else np.zeros_like(A)
    assert np.array_equal(np.isnan(_np(got[0])), np.isnan(loss)) and np.array_equal(np.isinf(_np(got[0])), np.isinf(loss))
    fine = np.isfinite(loss)
    err = np.abs(np.where(fine, _np(got[0]).astype(np.float64), 0) - np.where(fine, loss, 0))
    assert np.all(err[fine] <= (A * Z + 2 * r * Z + 2.0 ** -24 * np.abs(loss))[fine] + 1e-14), err.max()
    if got[1] is None:
        return
    g = _np(got[1]).astype(np.float64)
    with np.errstate(all="ignore"):
        x = l.astype(np.float64) / Tn[:, None, None]
        x -= x.max(-1, keepdims=True)
        s = np.exp(x)
        s /= s.sum(-1, keepdims=True)
        q = s / np.maximum(out, 1e-300)[..., None]
        per = (w / Tn[:, None])[..., None]
        bits = np.where(np.isfinite(x), -x / np.log(2), 0)
        Ar = (A + r)[..., None]
        tol = per * (Ar * s * 2 * Z + np.abs(Ar * out[..., None] - r[..., None]) * q * (Z + 2.0 ** -22 + 2.0 ** -23 + bits * np.log(2) * 2.0 ** -23))
        tol = np.where(n[..., None] > 0, tol, 0)        # an ignored row: exactly 0
        tol += np.abs(grad) * (2.0 ** -8 if logits.dtype == torch.bfloat16 else 2.0 ** -24) + 2.0 ** -126 * (1 + per)
    bad = np.isnan(grad)
    assert np.array_equal(np.isnan(g), bad)
    tol, diff = np.where(bad, 0, tol), np.where(bad, 0, np.abs(g - grad))
    assert np.all(diff <= tol), (np.max(diff - tol), np.unravel_index(np.argmax(diff - tol), diff.shape))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,R,V,K,pad,front", [
    (1, 1, 1, 1, 0, 0),                 # one token, one entry
    (2, 3, 2, 1, 0, 0),
    (3, 2, 7, 7, 0, 0),                 # every entry the teacher's: nothing outside
    (2, 5, 1000, 10, 3, 0),             # less than a chunk, padded rows
    (3, 3, 1025, 64, 0, 0),             # a chunk and one entry, rows at any offset
    (2, 2, 8192, 257, 8, 0),            # more entries than threads
    (1, 4, 32000, 32, 0, 0),
    (2, 2, 50381, 50, 5, 0),
    (2, 2, 50381, 50, 0, 1),            # the first row off its granule too
    (2, 3, 128256, 1024, 0, 0),
    (1, 3, 262144, 128, 0, 0),
])
def test_loss_and_gradient(ps, B, R, V, K, pad, front, dtype, tail):
    x = _inputs(B, R, V, K, dtype, V + K + tail, pad, total=0.83 if tail else None, front=front)
    ctx = ps.Context(1, 1, V, K)
    try:
        got = ctx.distill(*x[:5], weight=x[5], tail=tail)
        assert ctx.status(clear=True)[0] == 0
        _check(got, *x, tail)
        alone = ctx.distill(*x[:5], tail=tail, want_grad=False)
        assert torch.equal(alone[0], got[0]) and alone[1] is None
        only = ctx.distill(*x[:5], weight=x[5], tail=tail, want_loss=False)
        assert only[0] is None and torch.equal(only[1], got[1])
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype,V", [("bf16", 688120), ("f32", 344056), ("bf16", 400001)])
def test_the_longest_rows(ps, dtype, V):
    x = _inputs(1, 2, V, 5, dtype, V, total=0.9)
    ctx = ps.Context(1, 1, V, 8)
    try:
        _check(ctx.distill(*x[:5], weight=x[5], tail=True), *x, True)
        assert ctx.status(clear=True)[0] == 0
    finally:
        ctx.close()


def test_many_rows_and_few_give_the_same(ps):
    # how a row is spread over CTAs goes by the number of rows; a call gives the same however often it is made
    x = _inputs(1, 400, 9000, 20, "bf16", 5, total=0.7)
    ctx = ps.Context(1, 1, 9000, 20)
    try:
        got = ctx.distill(*x[:5], weight=x[5], tail=True)
        again = ctx.distill(*x[:5], weight=x[5], tail=True)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
        _check(got, *x, True)
        one = [x[0][:, :3], x[1], *[v[:, :3].contiguous() for v in x[2:]]]
        _check(ctx.distill(*one[:5], weight=one[5], tail=True), *one, True)
    finally:
        ctx.close()


@pytest.mark.parametrize("offset,spread", [(100.0, 2.0), (-300.0, 1.0), (0.0, 30.0), (0.0, 0.0), (3e4, 0.0)])
def test_offsets_and_peaked_rows(ps, offset, spread):
    # a common offset does not move a softmax; with a wide spread nearly all mass lies in one entry, inside or outside the teacher's
    x = _inputs(2, 3, 20000, 33, "f32", 9, offset=offset, spread=spread, total=0.6)
    ctx = ps.Context(1, 1, 20000, 64)
    try:
        for tail in (False, True):
            _check(ctx.distill(*x[:5], weight=x[5], tail=tail), *x, tail)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_student_holds_nearly_everything_in_the_entries(ps, dtype):
    # 1 - sum of s over the entries is 1e-9: its logarithm and the gradient outside the entries must still be right
    x = _inputs(2, 2, 30000, 40, dtype, 21, total=0.95)
    x[4].fill_(40)
    for b in range(2):
        for i in range(2):
            x[0][b, i, x[2][b, i].long()] += 36.0 * float(x[1][b])
    ctx = ps.Context(1, 1, 30000, 40)
    try:
        got = ctx.distill(*x[:5], weight=x[5], tail=True)
        assert rows.distill(_np(x[0]), _np(x[1]), _np(x[2]), _np(x[3]), _np(x[4]), None, True)[2].max() < 1e-8
        _check(got, *x, True)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_empty_rows_and_bad_data(ps, dtype):
    V, K = 10000, 6
    logits, T, idx, t, count, w = _inputs(4, 4, V, K, dtype, 31, total=0.9, pad=1)
    count.fill_(K)
    count[0, 0] = 0
    logits[0, 0] = float("nan")                         # an ignored row is not looked at
    logits[0, 1] = -float("inf")                        # one finite entry outside
    logits[0, 1, 77] = 1.0
    idx[0, 1, :] = torch.arange(6, device="cuda")
    logits[0, 2, idx[0, 2, 3].long()] = -float("inf")   # a teacher's entry that the student masks: an infinite loss
    logits[0, 3, 5000:] = torch.finfo(logits.dtype).min     # the type's lowest value as a mask
    T[3] = 1.0
    logits[1, 0, 9] = float("nan")
    logits[1, 1, int(idx[1, 1, 2])] = float("inf")
    logits[1, 2] = -float("inf")
    count[1, 3] = K + 1
    count[2, 0] = -1
    idx[2, 1, 2] = V
    idx[2, 2, 5] = idx[2, 2, 0]
    t[2, 3, 1] = float("nan")
    t[3, 0, 1] = -0.1
    idx[3, 1, 0] = -1
    t[3, 2, :] = 0.0                                    # nothing but zeros: without the tail a loss of 0
    t[3, 3, 0] = 0.0
    ctx = ps.Context(1, 1, V, K)
    try:
        for tail in (False, True):
            got = ctx.distill(logits, T, idx, t, count, weight=w, tail=tail)
            assert ctx.status(clear=True)[0] == 2 | 4
            _check(got, logits, T, idx, t, count, w, tail)
        assert float(got[0][0, 0]) == 0 and bool((got[1][0, 0] == 0).all())
        Tb = T.clone()
        Tb[2] = 0.0
        got = ctx.distill(logits, Tb, idx, t, count, weight=w)
        assert ctx.status(clear=True)[0] == 1 | 2 | 4 and bool(got[0][2].isnan().all())
        # nothing is written behind the rows
        assert bool(logits.as_strided((4, 4), (4 * (V + 1), V + 1), V).isnan().all())
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,pad", [(9000, 0), (9001, 0), (9001, 7)])
def test_the_gradient_in_place_of_the_logits_and_in_rows_of_its_own(ps, dtype, V, pad):
    x = _inputs(2, 9, V, 12, dtype, V + pad, pad)
    ctx = ps.Context(1, 1, V, 12)
    try:
        want = ctx.distill(*x[:5], weight=x[5])
        # another pitch than the logits', guarded
        buf = torch.full((2, 9, V + 11), 7.0, dtype=x[0].dtype, device="cuda")
        loss = torch.empty_like(want[0])
        ctx.distill(*x[:5], weight=x[5], out=(loss, buf[..., :V]))
        assert torch.equal(buf[..., :V], want[1]) and bool((buf[..., V:] == 7).all()) and torch.equal(loss, want[0])
        ctx.distill(*x[:5], weight=x[5], out=(loss, x[0]))
        assert torch.equal(x[0], want[1]) and torch.equal(loss, want[0])
    finally:
        ctx.close()


def test_autograd(ps):
    logits, T, idx, t, count, w = _inputs(2, 5, 5001, 20, "f32", 41, total=0.8)
    count[1, 1] = 0
    ctx = ps.Context(1, 1, 5001, 20)
    try:
        scale = torch.tensor(1.5, device="cuda", requires_grad=True)
        leaf = logits.clone().requires_grad_(True)
        loss = ctx.distill_loss(leaf * scale, T, idx, t, count, tail=True)
        (loss * w).sum().backward()
        got = ctx.distill((logits * 1.5).contiguous(), T, idx, t, count, weight=w, tail=True)
        assert torch.equal(loss.detach(), got[0])
        assert torch.equal(leaf.grad, got[1] * 1.5)
        assert leaf.grad[1, 1].abs().max() == 0
        # twice over the same graph, a sum's expanded gradient, no gradient wanted
        leaf2 = logits.clone().requires_grad_(True)
        loss = ctx.distill_loss(leaf2, T, idx, t, count)
        loss.sum().backward(retain_graph=True)
        first = leaf2.grad.clone()
        loss.sum().backward()
        assert torch.equal(leaf2.grad, 2 * first)
        assert not ctx.distill_loss(logits, T, idx, t, count).requires_grad
        with pytest.raises(RuntimeError):           # a second derivative is refused
            g, = torch.autograd.grad(ctx.distill_loss(leaf2, T, idx, t, count).sum(), leaf2, create_graph=True)
            g.sum().backward()
        with pytest.raises(RuntimeError):           # the logits were changed in between
            x = leaf2 * 1.0
            loss = ctx.distill_loss(x, T, idx, t, count)
            x.mul_(2)
            loss.sum().backward()
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_refusals(ps):
    logits, T, idx, t, count, w = _inputs(2, 3, 2000, 4, "bf16", 51)
    ctx = ps.Context(1, 1, 2000, 4)
    try:
        f = ctx.distill
        for args in [(logits.half(), T, idx, t, count), (logits[0], T, idx, t, count), (logits, T[:1], idx, t, count),
                     (logits, T.double(), idx, t, count), (logits, T, idx.long(), t, count),
                     (logits, T, idx, t[..., :2], count), (logits, T, idx, t.transpose(0, 1), count),
                     (logits, T, idx, t, count[:1]), (logits.cpu(), T, idx, t, count), (logits, T.cpu(), idx, t, count),
                     (logits.transpose(1, 2), T, idx, t, count), (logits, T, idx, t, None and count)]:
            with pytest.raises((ValueError, ps.PicospecError)):
                f(*args)
        with pytest.raises(ValueError):
            f(logits, T, idx, t, count, weight=w[:1])
        loss = torch.empty_like(w)
        with pytest.raises(ValueError):             # another type
            f(logits, T, idx, t, count, out=(loss, logits.float()))
        with pytest.raises(ValueError):
            f(logits, T, idx, t, count, out=(loss, logits[:, :2]))
        shared = torch.zeros(2 * 3 * 2000 + 8, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(ps.PicospecError):       # overlapping, but not the same place
            f(shared[:12000].view(2, 3, 2000), T, idx, t, count, out=(loss, shared[8:].view(2, 3, 2000)))
        with pytest.raises(ps.PicospecError):
            f(logits, T, idx, t, count, want_loss=False, want_grad=False)
        for V, k in ((2001, 4), (2000, 5)):
            z = torch.zeros((2, 3, k), dtype=torch.int32, device="cuda")
            with pytest.raises(ps.PicospecError) as e:
                f(torch.zeros((2, 3, V), device="cuda"), T, z, z.float(), count)
            assert e.value.code == -3
        big = ps.Context(1, 1, 500000, 4)
        with pytest.raises(ps.PicospecError) as e:  # a row beyond the shared memory of a cluster
            big.distill(torch.zeros((2, 3, 344057), device="cuda"), T, idx, t, count)
        assert e.value.code == -3
        big.close()
        empty = f(logits[:0], T[:0], idx[:0], t[:0], count[:0])
        assert empty[0].shape == (0, 3) and empty[1].shape == (0, 3, 2000)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_captured_replayed_and_on_other_streams(ps):
    x = _inputs(2, 40, 20000, 16, "bf16", 61)
    ctx = ps.Context(1, 1, 20000, 16)
    try:
        want = ctx.distill(*x[:5], weight=x[5])
        side = [torch.cuda.Stream() for _ in range(2)]
        outs = []
        for s in side:                              # two calls on one context at once
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append([ctx.distill(*x[:5], weight=x[5]) for _ in range(4)])
        torch.cuda.synchronize()
        for o in outs[0] + outs[1]:
            assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1])
        out = (torch.empty_like(want[0]), torch.empty_like(want[1]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.distill(*x[:5], weight=x[5], out=out)
        for _ in range(3):
            out[1].fill_(3)
            graph.replay()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        x[5].mul_(2)
        graph.replay()
        assert torch.equal(out[1], ctx.distill(*x[:5], weight=x[5])[1])
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_a_wait_that_runs_out_marks_the_rows(ps):
    x = _inputs(1, 3, 60000, 8, "bf16", 71)
    ctx = ps.Context(1, 1, 60000, 8)
    try:
        ctx.wait_limit(0)
        got = ctx.distill(*x[:5], weight=x[5])
        status = ctx.status(clear=True)[0]
        late = got[0].isnan()
        assert bool((got[1].isnan().all(-1) == late).all()) and (status == 8) == bool(late.any())
        ctx.wait_limit(2_000_000_000)
        _check(ctx.distill(*x[:5], weight=x[5]), *x, False)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype,N,V,K,tail", [
    ("bf16", 2100, 4099, 12, True),         # several rows a CTA; every row at another offset, tiles that some rows do not reach
    ("f32", 900, 8192, 300, False),         # more entries than threads
    ("bf16", 700, 33001, 40, False),        # clusters that take several rows
    ("f32", 420, 40001, 9, True),
])
def test_clusters_that_take_several_rows(ps, dtype, N, V, K, tail):
    # ignored, invalid and ordinary rows in turn: what one leaves behind (bits, barriers, records) must not reach the next
    x = list(_inputs(1, N, V, K, dtype, N + V, total=0.9))
    g = torch.Generator(device="cuda").manual_seed(N)
    kind = torch.randint(0, 10, (1, N), generator=g, device="cuda")
    x[4][kind == 0] = 0
    x[4][kind == 1] = -1
    x[4][:, -5:] = 0
    nan_rows = (kind == 2).nonzero()[:, 1]
    x[0][0, nan_rows, nan_rows % V] = float("nan")
    twice = (kind == 3).nonzero()[:, 1]
    x[4][0, twice] = K
    x[2][0, twice, 0] = x[2][0, twice, K - 1]
    ctx = ps.Context(1, 1, V, K)
    try:
        got = ctx.distill(*x[:5], weight=x[5], tail=tail)
        assert ctx.status(clear=True)[0] == 2 | 4
        _check(got, *x, tail)
        alone = ctx.distill(*x[:5], tail=tail, want_grad=False)[0]
        ctx.status(clear=True)
        assert torch.equal(alone.nan_to_num(-7.0), got[0].nan_to_num(-7.0))
        here = x[0].clone()
        ctx.distill(here, *x[1:5], weight=x[5], tail=tail, out=(torch.empty_like(alone), here))
        assert torch.equal(here.nan_to_num(-7.0), got[1].nan_to_num(-7.0))
    finally:
        ctx.close()


def test_late_waits_in_a_cluster_that_takes_several_rows(ps):
    x = _inputs(1, 1800, 6000, 8, "bf16", 73)
    ctx = ps.Context(1, 1, 6000, 8)
    try:
        want = ctx.distill(*x[:5], weight=x[5])
        ctx.wait_limit(0)
        got = ctx.distill(*x[:5], weight=x[5])
        status = ctx.status(clear=True)[0]
        late = got[0].isnan()
        assert (status == 8) == bool(late.any()) and bool((got[1].isnan().all(-1) == late).all())
        assert torch.equal(got[0][~late], want[0][~late]) and torch.equal(got[1][~late], want[1][~late])
        ctx.wait_limit(2_000_000_000)
        again = ctx.distill(*x[:5], weight=x[5])
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1]) and ctx.status()[0] == 0
    finally:
        ctx.close()
