"""Penalties, appends and gradient clipping without a GPU: the statements in oracle/rules.py against hand-made values, what autograd is told,
and what the library refuses before it touches a device."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rules
from paper_2603_19133_b200.binding import Context

EINVAL, ECUDA, ECAPACITY = -1, -2, -3


# ---- the statements -------------------------------------------------------------------------

def test_a_row_by_hand():
    # tokens: prompt 1, made 2 2 3, drafted 2; rho 2, frequency 0.5, presence 0.25, bias 1 on 4, 5 forbidden
    l = np.array([[[0.5, 3.0, -3.0, 4.0, 5.0, 9.0]] * 2])
    out = rules.penalize(l, history=np.array([[1, 2, 2, 3, 7]]), length=np.array([4]), prompt_length=np.array([1]), draft_tok=np.array([[2]]),
                         repetition=np.array([2.0]), presence=np.array([0.25]), frequency=np.array([0.5]),
                         bias=(np.array([[4, 0]]), np.array([[1.0, 7.0]]), np.array([1])), mask=np.array([[0b011111]]), mask_row=np.array([[0, -1]]))
    np.testing.assert_array_equal(out[0, 0], [0.5, 1.5, -6 - 1.0 - 0.25, 2 - 0.5 - 0.25, 6.0, -np.inf])
    np.testing.assert_array_equal(out[0, 1], [0.5, 1.5, -6 - 1.5 - 0.25, 2 - 0.5 - 0.25, 6.0, 9.0])


def test_the_gradient_is_that_of_the_rows():
    g = np.random.default_rng(0)
    B, R, V = 2, 3, 40
    x, w = 3 * g.standard_normal((B, R, V)), g.standard_normal((B, R, V))
    args = dict(history=g.integers(0, V, (B, 12)), length=np.array([12, 5]), prompt_length=np.array([3, 5]), draft_tok=g.integers(0, V, (B, R - 1)),
                repetition=np.array([1.4, 0.8]), presence=np.array([0.3, -0.1]), frequency=np.array([0.2, 0.4]),
                mask=g.integers(-2 ** 31, 2 ** 31, (4, 2)), mask_row=g.integers(-1, 4, (B, R)))
    grad = rules.penalize(x, **args, grad=w)
    h = 1e-6
    up, down = rules.penalize(x + h, **args), rules.penalize(x - h, **args)
    finite = np.isfinite(up)
    # (each side's sum is rounded at about 2^-50 of values below 2^5)
    np.testing.assert_allclose(grad[finite], ((up - down)[finite] / (2 * h)) * w[finite], atol=2.0 ** -44 / h)
    assert np.all(grad[~finite] == 0)


def test_appending_by_hand():
    history, length, bad = rules.append(np.zeros((3, 4), int), np.array([1, 2, 3]), np.array([9, 9, 9]), np.array([[1, 2]] * 3), np.array([1, -1, 2]))
    assert history.tolist() == [[0, 1, 9, 0], [0] * 4, [0] * 4] and length.tolist() == [3, 2, 3] and bad


def test_clipping_by_hand():
    norm, scale, out = rules.clip([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5.0 and scale == 0.2
    np.testing.assert_allclose(out[0], [0.6])
    assert rules.clip([np.array([np.inf])], 1.0)[1] == 1.0


# ---- autograd ---------------------------------------------------------------------------------

class Stand(Context):
    """A context whose rules scale by the repetition penalty."""

    def __init__(self):
        self.calls = []

    def penalize(self, logits, history=None, length=None, prompt_length=None, draft_tok=None, repetition=None, presence=None, frequency=None,
                 bias=None, mask=None, mask_row=None, out=None):
        self.calls.append("forward")
        return logits.detach() * (1.0 if repetition is None else repetition[:, None, None])

    def penalize_grad(self, grad, logits, history=None, length=None, prompt_length=None, draft_tok=None, repetition=None, presence=None,
                      frequency=None, bias=None, mask=None, mask_row=None, out=None):
        self.calls.append(("backward", logits is not None, history is not None, mask is not None, grad.is_contiguous()))
        return grad * (1.0 if repetition is None else repetition[:, None, None])


def test_the_logits_get_their_gradient():
    ctx, leaf, w = Stand(), torch.randn(2, 3, 7, requires_grad=True), torch.randn(2, 3, 7)
    rho, history = torch.tensor([2.0, 3.0]), torch.zeros(2, 4, dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    (ctx.penalized(leaf, history, n, repetition=rho) * w).sum().backward()
    torch.testing.assert_close(leaf.grad, w * rho[:, None, None])
    ctx.penalized(leaf, history, n, presence=rho, mask=torch.zeros(2, 3, 1, dtype=torch.int32)).sum().backward()
    # without a repetition penalty neither the logits nor the history are kept
    assert ctx.calls == ["forward", ("backward", True, True, False, True), "forward", ("backward", False, False, True, True)]
    with torch.no_grad():
        assert not ctx.penalized(leaf, history, n, repetition=rho).requires_grad


@pytest.mark.parametrize("name", ["repetition", "presence", "frequency", "bias"])
def test_rules_that_require_a_gradient_are_refused(name):
    ctx, leaf = Stand(), torch.randn(1, 1, 4, requires_grad=True)
    value = torch.ones(1, requires_grad=True)
    args = {"bias": (torch.zeros(1, 1, dtype=torch.int32), value.view(1, 1), torch.ones(1, dtype=torch.int32))} if name == "bias" else {name: value}
    with pytest.raises(ValueError, match=name):
        ctx.penalized(leaf, **args)
    with torch.no_grad():
        ctx.penalized(leaf, **args)


def test_tensors_of_the_host_are_refused():
    ctx = Context.__new__(Context)
    ctx._h, ctx.device = ctypes.c_void_p(), 0
    import paper_2603_19133_b200 as ps
    ps.lib()
    x = torch.zeros(1, 1, 8)
    for call in (lambda: ctx.penalize(x), lambda: ctx.penalize_grad(x, x), lambda: ctx.append(torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)),
                 lambda: ctx.grad_norm([x]), lambda: ctx.clip_grad([x], 1.0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="bias"):
        ctx.penalize(x, bias=(x, x))
    # what autograd would not see
    leaf = torch.zeros(1, 1, 8, requires_grad=True)
    for call in (lambda: ctx.penalize(leaf), lambda: ctx.penalize(x, out=leaf)):
        with pytest.raises(ValueError, match="autograd"):
            call()
    for call in (lambda: ctx.clip_grad([leaf], 1.0), lambda: ctx.clip_grad([x], 1.0, out=[leaf])):
        with pytest.raises(ValueError, match="requires a gradient|dense CUDA"):
            call()
    with pytest.raises(ValueError, match="requires a gradient"):
        ctx.clip_grad([leaf], 1.0)


# ---- refusals of the library, on a context that no device stands behind -------------------------

class Rules(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_stride", ctypes.c_longlong), ("capacity", ctypes.c_int), ("length", ctypes.c_void_p),
                ("prompt_length", ctypes.c_void_p), ("draft_tok", ctypes.c_void_p), ("repetition", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("frequency", ctypes.c_void_p), ("bias_idx", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("bias_count", ctypes.c_void_p),
                ("bias_k", ctypes.c_int), ("mask", ctypes.c_void_p), ("mask_stride", ctypes.c_longlong), ("mask_rows", ctypes.c_int),
                ("mask_row", ctypes.c_void_p)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_longlong), ("dtype", ctypes.c_int)]


@pytest.fixture()
def lib():
    if torch.cuda.is_available():
        pytest.skip("a call that passes the checks would reach the device")
    import paper_2603_19133_b200 as ps
    return ps.lib()


@pytest.fixture()
def fake(lib):
    # device, max_batch, max_gamma, max_vocab, max_k, SMs: the first members of a context
    buf = (ctypes.c_int * 65536)()
    buf[0], buf[1], buf[2], buf[3], buf[4], buf[5] = 0, 1, 1, 1000, 1, 148
    return ctypes.cast(buf, ctypes.c_void_p)


A, B_, W = 1 << 20, 1 << 30, 1 << 40          # addresses that are never looked at


def _penalize(lib, fake, rules, logits=A, dtype=1, B=2, R=3, V=1000, stride=1000, out=B_, out_stride=1000, work=W):
    return lib.picospec_penalize(fake, logits, dtype, B, R, V, stride, ctypes.byref(rules) if rules is not None else None, out, out_stride, work, None)


def test_penalize_checks_its_arguments(lib, fake):
    ok = dict(history=A, history_stride=10, capacity=10, length=A, repetition=A, bias_idx=A, bias=A, bias_count=A, bias_k=4, mask=A, mask_stride=32,
              mask_rows=5, mask_row=A)
    assert _penalize(lib, fake, Rules(**ok)) == ECUDA                  # all checks passed: there is no device
    assert _penalize(lib, fake, Rules()) == ECUDA and _penalize(lib, fake, Rules(), work=None) == ECUDA
    for change, code in [({"length": None}, EINVAL), ({"history_stride": 9}, EINVAL), ({"history_stride": -1}, EINVAL), ({"capacity": -1}, EINVAL),
                         ({"capacity": (1 << 27) + 1, "history_stride": 1 << 28}, ECAPACITY), ({"bias": None}, EINVAL), ({"bias_count": None}, EINVAL),
                         ({"bias_k": 0}, EINVAL), ({"bias_k": 1025}, ECAPACITY), ({"mask_rows": 0}, EINVAL), ({"mask_stride": 31}, EINVAL),
                         ({"mask_row": None}, EINVAL), ({"mask_row": None, "mask_rows": 6}, ECUDA), ({"history_stride": 0}, ECUDA),
                         ({"mask_stride": 0}, ECUDA), ({"repetition": None, "length": None}, ECUDA)]:
        assert _penalize(lib, fake, Rules(**{**ok, **change})) == code, change
    r = Rules(**ok)
    for change, code in [({"logits": None}, EINVAL), ({"out": None}, EINVAL), ({"dtype": 2}, EINVAL), ({"V": 0}, EINVAL), ({"V": 1001, "stride": 1001, "out_stride": 1001}, ECAPACITY),
                         ({"stride": 999}, EINVAL), ({"out_stride": 999}, EINVAL), ({"logits": A + 1}, EINVAL), ({"out": A + 2}, EINVAL), ({"out": A}, ECUDA),
                         ({"out": A, "out_stride": 1001}, EINVAL), ({"out": A + 2 * 5999}, EINVAL), ({"out": A + 2 * 6000}, ECUDA), ({"B": -1}, EINVAL),
                         ({"B": 1 << 27, "R": 2}, ECAPACITY), ({"work": None}, EINVAL), ({"work": W + 8}, EINVAL), ({"B": 0, "logits": None, "out": None}, 0),
                         ({"R": 0}, 0)]:
        assert _penalize(lib, fake, r, **change) == code, change
    assert _penalize(lib, None, r) == EINVAL and _penalize(lib, fake, None) == EINVAL

    def grad(rules, logits=W, out=B_):
        return lib.picospec_penalize_grad(fake, A, 1, 2, 3, 1000, 1000, logits, 1000, ctypes.byref(rules), out, 1000, W, None)
    assert grad(r) == ECUDA and grad(r, logits=None) == EINVAL and grad(r, out=W) == EINVAL and grad(r, out=A) == ECUDA
    assert grad(Rules(**{**ok, "repetition": None}), logits=None) == ECUDA


def test_the_workspace_holds_the_list(lib):
    size = lambda back=0, B=3, R=2, V=1000, **k: lib.picospec_rules_workspace(ctypes.byref(Rules(**k)), back, B, R, V)
    assert size() == 0 and size(mask=A, mask_rows=6, mask_stride=32) == 0
    h = dict(history=A, length=A, capacity=100, history_stride=100)
    one = size(**h, repetition=A)
    assert one >= 3 * 100 * 8 and size(**h, presence=A, back=1) == 0 and size(**h) == 0
    assert size(**h, repetition=A, bias_idx=A, bias=A, bias_count=A, bias_k=8) > one == size(**h, repetition=A, bias_idx=A, bias=A, bias_count=A, bias_k=8, back=1)
    assert size(**{**h, "capacity": 10 ** 6, "history_stride": 10 ** 6}, repetition=A) < 3 * 1000 * 8 + 200     # (never more than the vocabulary)
    assert size(**{**h, "capacity": -1}, repetition=A) == -1 and lib.picospec_rules_workspace(None, 0, 1, 1, 1) == -1


def test_append_checks_its_arguments(lib, fake):
    def call(history=A, stride=10, capacity=10, B=2, length=A, draft=A, G=3, accept=A, token=A, out=A, ctx=fake):
        return lib.picospec_append(ctx, history, stride, capacity, B, length, draft, G, accept, token, out, None)
    assert call() == ECUDA and call(draft=None, G=0, accept=None) == ECUDA and call(token=None) == ECUDA and call(B=0, history=None) == 0
    for change in [{"history": None}, {"length": None}, {"out": None}, {"stride": 9}, {"capacity": -1}, {"B": -1}, {"G": -1}, {"accept": None},
                   {"draft": None}, {"token": None, "accept": None, "draft": None, "G": 0}, {"ctx": None}]:
        assert call(**change) == EINVAL, change
    assert call(capacity=(1 << 27) + 1, stride=1 << 28) == ECAPACITY


def test_clipping_checks_its_arguments(lib, fake):
    def tensors(*specs):
        return (Tensor * max(1, len(specs)))(*[Tensor(*s) for s in specs])

    def clip(t, o=None, n=None, max_norm=1.0, norm_in=None, work=W, ctx=fake):
        return lib.picospec_clip_grad(ctx, t, o, len(t) if n is None else n, max_norm, norm_in, work, A, None)
    t = tensors((A, 10, 0), (B_, 20, 1))
    assert clip(t) == ECUDA and clip(t, max_norm=0.0) == ECUDA and clip(t, norm_in=A, work=None) == ECUDA
    assert clip(t, max_norm=-1.0) == clip(t, max_norm=float("nan")) == clip(t, work=None) == clip(t, work=W + 4) == clip(None, n=1) == clip(t, ctx=None) == EINVAL
    assert clip(t, n=-1) == EINVAL and clip(tensors((A, -1, 0))) == EINVAL and clip(tensors((A, 1, 2))) == EINVAL
    assert clip(tensors((None, 1, 0))) == EINVAL and clip(tensors((None, 0, 0))) == ECUDA and clip(tensors((A + 2, 1, 0))) == EINVAL
    assert clip(tensors((A + 2, 1, 1))) == ECUDA and clip(tensors((A, 1 << 40, 1))) == ECAPACITY
    # overlaps: what is written overlaps nothing else
    assert clip(tensors((A, 10, 0), (A + 36, 10, 0))) == EINVAL and clip(tensors((A, 10, 0), (A + 40, 10, 0))) == ECUDA
    assert clip(tensors((A + 40, 10, 0), (A, 10, 0))) == ECUDA and clip(tensors((A, 10, 0), (A, 10, 0))) == EINVAL
    assert clip(t, tensors((W, 10, 0), (W + 40, 20, 1))) == ECUDA and clip(t, t) == ECUDA
    assert clip(t, tensors((W, 10, 0), (W + 36, 20, 1))) == EINVAL and clip(t, tensors((W, 10, 0), (A, 20, 1))) == EINVAL
    assert clip(t, tensors((A + 4, 10, 0), (W, 20, 1))) == EINVAL and clip(t, tensors((W, 11, 0), (W + 64, 20, 1))) == EINVAL
    assert clip(tensors((A, 10, 0), (A, 10, 0)), tensors((W, 10, 0), (W + 40, 10, 0))) == ECUDA        # (read twice, written once)
    assert lib.picospec_grad_norm(fake, t, 2, W, A, None) == ECUDA and lib.picospec_grad_norm(fake, t, 2, None, A, None) == EINVAL
    assert lib.picospec_grad_norm(fake, t, 2, W, None, None) == EINVAL and lib.picospec_grad_norm(fake, None, 0, W, A, None) == ECUDA
    assert lib.picospec_grad_workspace(1) == lib.picospec_grad_workspace(1024) < lib.picospec_grad_workspace(1025)
