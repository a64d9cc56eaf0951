"""The double-precision statements of the operators on dense rows, pinned without a GPU: against differences,
closed forms and brute force."""
import numpy as np
import pytest

from oracle import rows


def _case(rng, V, K, B=2, R=2, total=0.8):
    l = rng.normal(size=(B, R, V)) * 2
    idx = np.stack([[rng.permutation(V)[:K] for _ in range(R)] for _ in range(B)]).astype(np.int32)
    t = rng.random((B, R, K))
    t *= total / t.sum(-1, keepdims=True)
    return l, rng.uniform(0.5, 1.5, B), idx, t, np.full((B, R), K, np.int32), rng.random((B, R)) + 0.1


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,K,total", [(2, 1, 0.7), (7, 3, 1.0), (40, 12, 0.9), (9, 8, 0.5)])
def test_distill_gradient_is_the_losses_difference(V, K, total, tail):
    rng = np.random.default_rng(V + K)
    l, T, idx, t, n, w = _case(rng, V, K, total=total)
    loss, grad, _ = rows.distill(l, T, idx, t, n, w, tail)
    h = 1e-5
    for v in range(V):
        up, down = l.copy(), l.copy()
        up[..., v] += h
        down[..., v] -= h
        d = (rows.distill(up, T, idx, t, n, None, tail)[0] - rows.distill(down, T, idx, t, n, None, tail)[0]) / (2 * h)
        # central differences: h^2 times a third derivative of at most 2 / T^3 <= 16, and 2^-52 |loss| / h
        np.testing.assert_allclose(grad[..., v], w * d, rtol=0, atol=16 * h * h + 1e-9)


def test_distill_closed_forms():
    rng = np.random.default_rng(3)
    V, K = 12, 12
    l, T, _, _, n, _ = _case(rng, V, K)
    idx = np.broadcast_to(np.arange(V, dtype=np.int32), (2, 2, V)).copy()
    x = l / T[:, None, None]
    s = np.exp(x - x.max(-1, keepdims=True))
    s /= s.sum(-1, keepdims=True)
    loss, grad, _ = rows.distill(l, T, idx, s, n)              # the student is the teacher
    np.testing.assert_allclose(loss, 0, atol=1e-14)
    np.testing.assert_allclose(grad, 0, atol=1e-15)
    one = np.zeros_like(s)
    one[..., 4] = 1.0                                          # one certain outcome: the cross-entropy
    loss, grad, _ = rows.distill(l, T, idx, one, n)
    np.testing.assert_allclose(loss, -np.log(s[..., 4]), rtol=1e-12)
    np.testing.assert_allclose(grad, (s - one) / T[:, None, None], rtol=1e-12, atol=1e-15)
    # half of the teacher given, the rest as one outcome: the same entries merged into one by hand
    half = idx[..., :6]
    loss, grad, out = rows.distill(l, T, half, s[..., :6] * 0.9, n * 0 + 6, tail=True)
    t, r = s[..., :6] * 0.9, 1 - 0.9 * s[..., :6].sum(-1)
    want = (t * np.log(0.9)).sum(-1) + r * np.log(r / s[..., 6:].sum(-1))
    np.testing.assert_allclose(loss, want, rtol=1e-10, atol=1e-13)
    np.testing.assert_allclose(out, s[..., 6:].sum(-1), rtol=1e-12)
    assert np.all(np.abs(grad.sum(-1)) < 1e-14)                # a softmax does not see a common offset


def test_distill_special_rows():
    l = np.zeros((1, 6, 5))
    l[0, 1, 2] = -np.inf
    l[0, 2, 0] = np.nan
    idx = np.tile(np.array([2, 4], np.int32), (1, 6, 1))
    t = np.full((1, 6, 2), 0.5)
    n = np.array([[0, 2, 2, 3, 2, 2]], np.int32)
    idx[0, 4] = [3, 3]
    t[0, 5] = [0.0, 1.0]
    loss, grad, _ = rows.distill(l, np.ones(1), idx, t, n)
    assert loss[0, 0] == 0 and np.all(grad[0, 0] == 0)
    assert loss[0, 1] == np.inf and np.all(np.isfinite(grad[0, 1])) and grad[0, 1, 2] == -0.5
    assert np.isnan(loss[0, 2]) and np.isnan(loss[0, 3]) and np.isnan(loss[0, 4]) and np.all(np.isnan(grad[0, 2:5]))
    assert np.isclose(loss[0, 5], np.log(5))


def test_sample_keeps_what_the_limits_say():
    # by hand: weights 8 4 4 2 1 1 of Z = 20, in an order that is not the vocabulary's
    w = np.array([1.0, 4.0, 8.0, 2.0, 4.0, 1.0])
    l = np.log(w)[None, None]
    u, one = np.zeros((1, 1, 2)), np.ones(1)

    def count(**limits):
        return int(rows.sample(l, one, u, **{n: np.array([v]) for n, v in limits.items()})[3][0, 0])

    assert count() == 6 and count(top_k=0) == 6 and count(top_k=4) == 4 and count(top_k=9) == 6
    assert [count(top_p=x) for x in (0.1, 0.4 - 1e-12, 0.4 + 1e-12, 0.8 - 1e-12, 0.8 + 1e-12, 0.9 + 1e-12, 0.95 + 1e-12, 1.0)] == [1, 1, 2, 3, 4, 5, 6, 6]
    assert [count(min_p=x) for x in (0.0, 0.125 - 1e-12, 0.125 + 1e-12, 0.5 - 1e-12, 0.6, 1.0)] == [6, 6, 4, 3, 1, 1]
    assert count(top_k=4, top_p=0.7, min_p=0.1) == 3 and count(top_k=2, top_p=0.7, min_p=0.1) == 2
    token = rows.sample(l, one, u, top_k=np.array([1]))[0]
    assert token[0, 0] == 2
    tie = rows.sample(l, one, np.full((1, 1, 2), 0.999), top_k=np.array([2]))       # of the two 4s the lower index
    assert tie[0][0, 0] == 2 and rows.sample(l, one, u, top_k=np.array([2]))[0][0, 0] == 1


@pytest.mark.parametrize("limits", [{}, {"top_k": 3}, {"top_p": 0.7}, {"min_p": 0.3}, {"top_k": 5, "top_p": 0.9, "min_p": 0.05}])
def test_sample_law(limits):
    # over a grid of uniforms the share of a token is its probability among the kept ones
    rng = np.random.default_rng(5)
    l, T = rng.normal(size=(1, 1, 9)) * 1.5, 0.8
    n = 200
    g = (np.arange(n) + 0.5) / n
    u = np.stack(np.meshgrid(g, g, indexing="ij"), -1).reshape(n * n, 1, 2)
    full = {k: np.full(n * n, v) for k, v in limits.items()}
    token, prob, logprob, count = rows.sample(np.broadcast_to(l, (n * n, 1, 9)), np.full(n * n, T), u, chunk=4, **full)
    q = np.exp(l[0, 0] / T)
    order = np.argsort(-q)
    keep = order[:count[0, 0]]
    law = np.zeros(9)
    law[keep] = q[keep] / q[keep].sum()
    got = np.bincount(token[:, 0], minlength=9) / (n * n)
    assert np.all(got[law == 0] == 0)
    np.testing.assert_allclose(got, law, atol=2 / n)            # each of the two levels off by at most a step of the grid
    np.testing.assert_allclose(prob[:, 0], law[token[:, 0]], rtol=1e-12)
    np.testing.assert_allclose(logprob[:, 0], np.log(q / q.sum())[token[:, 0]], rtol=1e-10)


@pytest.mark.parametrize("top", [2.0, -40.0, 3e38, -3e38])
def test_distill_counts_entries_that_share_the_largest_logit(top):
    # n entries share the largest logit, all others are far below: s = 1 / n on each of them, however large the logit
    V, n = 50, 5
    l = np.full((1, 1, V), top - max(1.0, abs(top)) * 1e3 / 64)
    l[..., 3:3 + n] = top
    idx, t = np.array([[[3, 4]]], np.int32), np.array([[[0.25, 0.5]]])
    loss, grad, out = rows.distill(l, np.array([0.01]), idx, t, np.array([[2]]), None, True)
    # ln R = ln(3 / 5);  r = 1/4
    want = 0.25 * np.log(0.25 * n) + 0.5 * np.log(0.5 * n) + 0.25 * (np.log(0.25) - np.log(3 / n))
    np.testing.assert_allclose(loss, want, rtol=1e-13)
    np.testing.assert_allclose(out, 3 / n, rtol=1e-13)
    g = np.zeros(V)
    g[3:3 + n] = 1 / n
    g[3], g[4] = g[3] - 0.25, g[4] - 0.5
    g[5:3 + n] -= 0.25 / 3
    np.testing.assert_allclose(grad[0, 0], g / 0.01, rtol=1e-12, atol=1e-12)


def test_sample_min_p_next_to_one():
    # weights 1 - 1e-17 .. are 1 in double precision; min_p = 1 keeps those that are
    l = np.array([1.0, 1.0 - 2.0 ** -30, 1.0, 0.5])[None, None]
    u, T = np.zeros((1, 1, 2)), np.array([1e12])
    for m, kept in ((1.0, 2), (1 - 2.0 ** -53, 3), (1 - 1e-12, 4)):
        assert rows.sample(l, T, u, min_p=np.array([m]))[3][0, 0] == kept


@pytest.mark.parametrize("far", [20.0, 1e18, 3e38])
def test_distill_outside_the_entries_beside_a_far_one(far):
    # one entry holds everything; the rest is a softmax of its own, and its gradient is -r times that
    l = np.array([far, 1.0, 2.0, 3.0, -np.inf])[None, None]
    loss, grad, out = rows.distill(l, np.array([0.5]), np.array([[[0]]], np.int32), np.array([[[0.75]]]), np.array([[1]]), None, True)
    q = np.exp(np.array([2.0, 4.0, 6.0, -np.inf]))
    share = q.sum() / (q.sum() + np.exp(2 * far)) if far < 100 else 0.0
    # ((A + r) R - r) / R * s, on the scale of the complement's softmax; A + r = 1
    np.testing.assert_allclose(grad[0, 0, 1:], (share - 0.25) * q / q.sum() / 0.5, rtol=1e-12)
    np.testing.assert_allclose(out, share, rtol=1e-12)
    want = 0.75 * np.log(0.75) + 0.25 * np.log(0.25) - 0.75 * np.log1p(-share) - 0.25 * (6.0 - 2 * far + np.log(np.exp([-4.0, -2.0, 0.0]).sum()) + np.log1p(-share))
    np.testing.assert_allclose(loss, want, rtol=1e-13)
