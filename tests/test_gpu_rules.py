"""Penalties, biases and masks on rows of logits, and their gradient, against the double-precision statement (oracle/rules.py).  The kernel
computes in double precision and rounds once: half a step of the type, 2^-24 or 2^-8 relative (half of the smallest subnormal where the
value is that small), and the double-precision products and differences before it, a few 2^-53 of the largest of the terms (TERMS of at most 2^10
here).  Entries that no rule concerns keep their bits."""
import numpy as np
import pytest
import torch

from oracle import rules as oracle

pytestmark = pytest.mark.gpu

RTOL = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
ATOL = 8 * 2.0 ** -53 * 2.0 ** 10
NAMES = ("history", "length", "prompt_length", "draft_tok", "repetition", "presence", "frequency", "bias", "mask", "mask_row")


@pytest.fixture(scope="module")
def ps():
    import paper_2603_19133_b200 as ps
    ps.lib()
    return ps


@pytest.fixture()
def ctx(ps):
    c = ps.Context(1, 1, 1 << 20, 1)
    yield c
    c.close()


def _np(t):
    if isinstance(t, tuple):
        return tuple(_np(x) for x in t)
    if t is None:
        return None
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def _stored(values, dtype, pad=0, front=0):
    """In rows of V + pad elements (NaN between them) that start `front` elements late."""
    B, R, V = values.shape
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((B * R * (V + pad) + front + 8,), float("nan"), dtype=td, device="cuda")
    rows = buf[front:front + B * R * (V + pad)].view(B, R, V + pad)[..., :V]
    rows.copy_(values)
    return rows


def _rules(B, R, V, L, law, seed, K=7, M=5):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(hi, *shape):
        return torch.randint(0, hi, shape, generator=g, device="cuda", dtype=torch.int32)

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    out = {}
    if "h" in law:
        # few different tokens: most come several times
        out["history"] = (ints(V, B, L).double() * rand(B, L) ** 3).to(torch.int32)
        out["length"] = ints(L + 1, B)
        out["length"][0] = L
        if B > 2:
            out["length"][1], out["length"][2] = 0, min(1, L)
        out["prompt_length"] = torch.minimum(ints(L + 1, B), out["length"])
    if "d" in law and R > 1:
        out["draft_tok"] = (ints(V, B, R - 1).double() * rand(B, R - 1) ** 3).to(torch.int32)
    if "r" in law:
        out["repetition"] = 0.7 + 0.6 * rand(B)
    if "p" in law:
        out["presence"] = 2 * rand(B) - 0.5
    if "f" in law:
        out["frequency"] = rand(B) - 0.3
    if "b" in law:
        K = min(K, V)
        idx = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(B)]).to(torch.int32)
        out["bias"] = (idx, 20 * torch.randn((B, K), generator=g, device="cuda"), ints(K + 1, B))
        out["bias"][1][:, 0] = -float("inf")
    if "m" in law or "M" in law:
        W = (V + 31) // 32
        shape = (M, W) if "m" in law else (B, R, W)
        words = torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device="cuda", dtype=torch.int64)
        words |= torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device="cuda", dtype=torch.int64)
        few = torch.where(torch.rand(shape, generator=g, device="cuda") < 0.1, 1 << torch.randint(0, 32, shape, generator=g, device="cuda"), 0)
        few = torch.where(few >= 1 << 31, few - (1 << 32), few)
        kind = torch.randint(0, 5, shape[:-1], generator=g, device="cuda")[..., None]
        words = torch.where(kind == 1, -1, torch.where(kind == 2, 0, torch.where(kind == 3, few, words)))       # all, none, few, three in four
        out["mask"] = words.to(torch.int32)
        if "m" in law:
            out["mask_row"] = ints(M + 1, B, R) - 1
    return out


def _logits(B, R, V, dtype, seed, pad=0, front=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = 4 * torch.randn((B, R, V), generator=g, device="cuda")
    return _stored(x, dtype, pad, front)


def _check(got, want, source, dtype, changed=None):
    """`source`: what an entry that no rule concerns has to equal, bit by bit."""
    got_np = _np(got).astype(np.float64)
    assert np.array_equal(np.isnan(got_np), np.isnan(want))
    np.testing.assert_allclose(got_np, want, rtol=RTOL[dtype], atol=ATOL)
    if changed is not None:
        same = torch.from_numpy(~changed).to(got.device)
        assert torch.equal(_bits(got)[same], _bits(source)[same])


def _changed(rules, B, R, V):
    """Entries that a rule concerns: what a row of ones and one of minus ones do not come out of alike, or any bias or mask."""
    out = np.zeros((B, R, V), bool)
    if rules.get("history") is not None or rules.get("draft_tok") is not None:
        for b in range(B):
            n = int(rules["length"][b]) if "length" in rules else 0
            seen = np.zeros(V, bool)
            seen[_np(rules["history"][b, :n]) if n else []] = True
            for i in range(R):
                if i and "draft_tok" in rules:
                    seen[int(rules["draft_tok"][b, i - 1])] = True
                out[b, i] |= seen
    if "bias" in rules:
        for b in range(B):
            out[b][:, _np(rules["bias"][0][b, :int(rules["bias"][2][b])])] = True
    return out


SHAPES = [  # B, R, V, L, dtype, pad, front
    (1, 1, 1, 1, "f32", 0, 0),
    (1, 1, 31, 5, "bf16", 0, 0),
    (3, 2, 33, 0, "bf16", 0, 0),
    (2, 3, 1000, 40, "f32", 0, 0),
    (3, 4, 1003, 77, "bf16", 0, 0),             # the offset changes from row to row
    (3, 5, 8192, 300, "bf16", 0, 0),
    (2, 2, 8193, 1001, "bf16", 7, 0),
    (2, 3, 9001, 700, "f32", 3, 1),             # every offset from a boundary
    (2, 3, 9001, 700, "bf16", 0, 5),
    (1, 9, 50381, 5000, "bf16", 3, 0),
    (4, 1, 32000, 513, "f32", 0, 0),
    (1, 40, 2049, 64, "bf16", 0, 0),            # more rows than a CTA takes
    (1, 35, 700, 9, "f32", 0, 0),
    # histories that a kernel of its own puts together
    (2, 5, 12001, 6000, "bf16", 3, 1),
    (2, 3, 9001, 5000, "f32", 0, 0),
    (1, 150, 5000, 6000, "bf16", 0, 0),         # many drafted tokens before a CTA's rows, more concerned entries than are counted beforehand
    (20, 1, 40000, 9000, "bf16", 0, 0),
]


@pytest.mark.parametrize("law", ["hr", "hpf", "hdrpf", "dr", "b", "m", "M", "hdrpfbm"])
@pytest.mark.parametrize("B,R,V,L,dtype,pad,front", SHAPES)
def test_forward(ctx, B, R, V, L, dtype, pad, front, law):
    x = _logits(B, R, V, dtype, V + L, pad, front)
    rules = _rules(B, R, V, L, law, 3 * V + L)
    want = oracle.penalize(_np(x), **{n: _np(v) for n, v in rules.items()})
    changed = _changed(rules, B, R, V) | np.isinf(want)
    got = ctx.penalize(x, **rules)
    _check(got, want, x, dtype, changed)
    # into rows at another offset, and in place
    other = _stored(torch.zeros((B, R, V)), dtype, pad + 1, front + 1)
    assert torch.equal(_bits(ctx.penalize(x, **rules, out=other)), _bits(got))
    place = _stored(x, dtype, pad, front)
    around = place.untyped_storage()
    assert ctx.penalize(place, **rules, out=place) is place
    assert torch.equal(_bits(place), _bits(got))
    if pad:     # what lies between the rows is left alone
        flat = torch.tensor([], dtype=x.dtype, device="cuda").set_(around)[front:front + B * R * (V + pad)].view(B, R, V + pad)
        assert bool(flat[..., V:].isnan().all())
    assert ctx.status()[0] == 0


@pytest.mark.parametrize("law", ["hdr", "hdrpfbm", "pfM", "dr"])
@pytest.mark.parametrize("B,R,V,L,dtype,pad,front", SHAPES)
def test_gradient(ctx, B, R, V, L, dtype, pad, front, law):
    x, g = _logits(B, R, V, dtype, V + L, pad, front), _logits(B, R, V, dtype, V + L + 1, 0, 0)
    rules = _rules(B, R, V, L, law, 3 * V + L)
    want = oracle.penalize(_np(x), **{n: _np(v) for n, v in rules.items()}, grad=_np(g))
    logits = x if "repetition" in rules else None
    got = ctx.penalize_grad(g, logits, **rules)
    _check(got, want, g, dtype)
    other = _stored(torch.zeros((B, R, V)), dtype, pad + 1, front + 1)
    assert torch.equal(_bits(ctx.penalize_grad(g, logits, **rules, out=other)), _bits(got))
    place = g.clone()
    assert torch.equal(_bits(ctx.penalize_grad(place, logits, **rules, out=place)), _bits(got))
    assert ctx.status()[0] == 0


@pytest.mark.parametrize("law", ["hdrpfbm", "r", "rb"])
def test_gradient_against_differences(ctx, law):
    # fp32 logits away from 0 by more than the step: y is linear there, and a step of 2^-6 moves y by rho * 2^-6; both sides of the difference are
    # rounded to 2^-24 of values below 2^7, so the quotient is off by 2 * 2^-18 / 2^-6 at most
    B, R, V = 2, 3, 400
    x = _logits(B, R, V, "f32", 5)
    x += torch.sign(x) * 0.25
    rules = _rules(B, R, V, 60, "h" + law if "h" not in law else law, 6)
    w = torch.randn((B, R, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(7))
    got = ctx.penalize_grad(w, x, **rules).double()
    up, down = ctx.penalize(x + 2.0 ** -7, **rules).double(), ctx.penalize(x - 2.0 ** -7, **rules).double()
    quotient = (up - down) * 2.0 ** 6
    quotient[~torch.isfinite(up)] = 0.0
    torch.testing.assert_close(got[torch.isfinite(up)], (quotient * w.double())[torch.isfinite(up)], rtol=2.0 ** -23,
                               atol=2 * 2.0 ** -18 * 2.0 ** 6 * float(w.abs().max()))
    masked = ~torch.isfinite(up) if "mask" in rules else torch.zeros_like(up, dtype=torch.bool)
    if "bias" not in rules:
        assert bool((got[masked] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_values(ctx, dtype):
    # infinities, NaN, zeros of either sign and the type's lowest value at seen, biased, masked and free places
    specials = [float("inf"), -float("inf"), float("nan"), 0.0, -0.0, -3.0e38, 3.0e38, 1e-40, -1e-40, 2.5]
    n = len(specials)
    x = torch.tensor(specials * 4, device="cuda").view(1, 1, 4 * n)
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    V = 4 * n
    at = torch.arange(V, device="cuda", dtype=torch.int32)
    mask = torch.zeros((1, 2), dtype=torch.int64)
    for v in range(3 * n):
        mask[0, v // 32] |= 1 << (v % 32)
    mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask).to(torch.int32).cuda()
    rules = dict(history=at[None, :n].contiguous(), length=torch.tensor([n], dtype=torch.int32, device="cuda"),
                 prompt_length=torch.tensor([n // 2], dtype=torch.int32, device="cuda"),
                 repetition=torch.tensor([1.25], device="cuda"), presence=torch.tensor([0.5], device="cuda"),
                 frequency=torch.tensor([0.25], device="cuda"),
                 bias=(at[None, n:2 * n].contiguous(), torch.full((1, n), -1.5, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")),
                 mask=mask, mask_row=torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    want = oracle.penalize(_np(x), **{k: _np(v) for k, v in rules.items()})[0, 0]
    got = ctx.penalize(x, **rules)
    tiny = torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps       # (a subnormal's step)
    with np.errstate(over="ignore"):
        limit = float(torch.finfo(x.dtype).max) * (1 + RTOL[dtype])
        want = np.where(np.abs(want) >= limit, np.copysign(np.inf, want), want)
    out = _np(got)[0, 0].astype(np.float64)
    assert np.array_equal(np.isnan(out), np.isnan(want))
    np.testing.assert_allclose(out, want, rtol=RTOL[dtype], atol=max(ATOL, 0.5 * tiny))
    assert torch.equal(_bits(got)[0, 0, 2 * n:3 * n], _bits(x)[0, 0, 2 * n:3 * n])        # free: bit by bit
    assert bool((got[0, 0, 3 * n:] == -float("inf")).all())                               # masked, whatever stood there
    grad = ctx.penalize_grad(x, x, **rules)
    assert bool((grad[0, 0, 3 * n:] == 0).all())
    assert ctx.status()[0] == 0


def test_an_index_that_comes_twice(ctx):
    # in a history it counts twice, in a list of biases the last one counts -- whichever thread comes first
    V, K = 5000, 1024
    x = torch.zeros((1, 1, V), device="cuda")
    idx = torch.randint(0, 40, (1, K), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    value = torch.arange(1, K + 1, device="cuda", dtype=torch.float32)[None]
    last = {int(v): j for j, v in enumerate(idx[0].tolist())}
    for _ in range(5):
        got = ctx.penalize(x, bias=(idx, value, torch.tensor([K], dtype=torch.int32, device="cuda")))[0, 0]
        assert all(float(got[v]) == j + 1 for v, j in last.items()) and int((got != 0).sum()) == len(last)
    history = torch.full((1, 3000), 17, dtype=torch.int32, device="cuda")
    got = ctx.penalize(x, history, torch.tensor([3000], dtype=torch.int32, device="cuda"), torch.tensor([1000], dtype=torch.int32, device="cuda"),
                       frequency=torch.ones(1, device="cuda"))
    assert float(got[0, 0, 17]) == -2000 and int((got != 0).sum()) == 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bad_data_marks_the_rows_concerned(ctx, dtype):
    B, R, V, L = 12, 3, 9000, 50
    nan = float("nan")
    for backward in (False, True):
        x = _logits(B, R, V, dtype, 1)
        rules = _rules(B, R, V, L, "hdrpfbm", 2)
        rules["length"][:] = L
        rules["prompt_length"][:] = 10
        rules["bias"][2][:] = 5
        rules["length"][0] = L + 1
        rules["length"][1] = -1
        rules["prompt_length"][2] = L + 1
        rules["history"][3, L - 1] = V
        rules["history"][4, 0] = -1
        rules["draft_tok"][5, 1] = V                    # the last row alone
        rules["repetition"][6] = 0.0
        rules["bias"][0][7, 4] = V
        rules["bias"][0][8, 5] = -7                     # behind the count
        rules["bias"][1][9, 2] = nan
        rules["mask_row"][10, 1] = 5                    # that row alone
        rules["frequency"][11] = float("inf")
        args = {n: _np(v) for n, v in rules.items()}
        if backward:
            g = _logits(B, R, V, dtype, 3)
            want, got = oracle.penalize(_np(x), **args, grad=_np(g)), ctx.penalize_grad(g, x, **rules)
        else:
            want, got = oracle.penalize(_np(x), **args), ctx.penalize(x, **rules)
        rows = np.isnan(want).all(-1)
        assert rows[:5].all() and not rows[5, 0] and rows[5, 2] and rows[6].all() and not rows[8].any() and rows[10].tolist() == [False, True, False]
        assert rows[7].all() == rows[9].all() == rows[11].all() == (not backward)
        assert np.array_equal(_np(got.isnan().all(-1)), rows)
        _check(got, want, x, dtype)
        assert ctx.status(clear=True)[0] == 4
        place = (g if backward else x).clone()
        if backward:
            ctx.penalize_grad(place, x, **rules, out=place)
        else:
            ctx.penalize(place, **rules, out=place)
        assert torch.equal(_bits(place), _bits(got)) and ctx.status(clear=True)[0] == 4
    # what is not read is not judged: the same history beside a mask alone
    ctx.penalize(x, rules["history"], rules["length"], mask=rules["mask"], mask_row=rules["mask_row"].clamp(max=4))
    assert ctx.status()[0] == 0


def test_a_mask_that_allows_nothing_and_one_that_allows_everything(ctx):
    V = 4099
    x = _logits(2, 2, V, "bf16", 1)
    mask = torch.stack([torch.zeros(129, dtype=torch.int32), torch.full((129,), -1, dtype=torch.int32)]).cuda()
    row = torch.tensor([[0, 1], [-1, 0]], dtype=torch.int32, device="cuda")
    got = ctx.penalize(x, mask=mask, mask_row=row)
    assert bool((got[0, 0] == -float("inf")).all()) and bool((got[1, 1] == -float("inf")).all())
    assert torch.equal(got[0, 1], x[0, 1]) and torch.equal(got[1, 0], x[1, 0])
    # the call that takes a row without an entry says so
    ctx.sample(got, torch.ones(2, device="cuda"), torch.rand((2, 2, 2), device="cuda"))
    assert ctx.status(clear=True)[0] == 2


def test_no_rules_at_all_and_empty_batches(ctx):
    x = _logits(2, 3, 777, "bf16", 1)
    assert torch.equal(ctx.penalize(x), x) and torch.equal(ctx.penalize_grad(x, None), x)
    for shape in ((0, 3, 777), (2, 0, 777)):
        e = torch.empty(shape, device="cuda")
        assert ctx.penalize(e).shape == shape
    # penalties without any history, a history without a place
    one = torch.ones(2, device="cuda")
    assert torch.equal(ctx.penalize(x, repetition=2 * one, presence=one), x)
    nothing = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    assert torch.equal(ctx.penalize(x, nothing, torch.zeros(2, dtype=torch.int32, device="cuda"), repetition=2 * one), x)
    assert ctx.status()[0] == 0
    assert bool(ctx.penalize(x, nothing, torch.ones(2, dtype=torch.int32, device="cuda"), repetition=2 * one).isnan().all())
    assert ctx.status(clear=True)[0] == 4


def test_broadcast_rows(ctx):
    # one history and one mask for all sequences, without copies of them
    B, R, V = 5, 2, 3001
    x = _logits(B, R, V, "f32", 4)
    rules = _rules(1, R, V, 90, "hm", 5, M=1)
    shared = dict(history=rules["history"].expand(B, -1), length=rules["length"].expand(B).contiguous(), repetition=torch.full((B,), 1.5, device="cuda"),
                  mask=rules["mask"].expand(3, -1), mask_row=torch.full((B, R), 2, dtype=torch.int32, device="cuda"))
    got = ctx.penalize(x, **shared)
    for b in range(B):
        alone = ctx.penalize(x[b:b + 1], rules["history"], rules["length"], repetition=torch.full((1,), 1.5, device="cuda"), mask=rules["mask"],
                             mask_row=torch.zeros((1, R), dtype=torch.int32, device="cuda"))
        assert torch.equal(got[b:b + 1], alone)


def test_offsets_beyond_32_bits(ctx):
    # rows of logits and of history that start more than 2^31 entries behind the first
    V, L, pitch = 5000, 300, 1 << 30
    logits = torch.empty(2 * pitch + V, dtype=torch.bfloat16, device="cuda").as_strided((3, 1, V), (pitch, pitch, 1))
    history = torch.empty(2 * pitch + L, dtype=torch.int32, device="cuda").as_strided((3, L), (pitch, 1))
    x, rules = _logits(3, 1, V, "bf16", 8), _rules(3, 1, V, L, "hrpf", 9)
    rules["length"][:] = L
    logits.copy_(x)
    history.copy_(rules["history"])
    got = ctx.penalize(logits, **{**rules, "history": history}, out=logits)
    assert torch.equal(got, ctx.penalize(x, **rules)) and ctx.status()[0] == 0


def test_a_long_history(ctx):
    B, R, V, L = 2, 3, 128256, 131072
    x, rules = _logits(B, R, V, "bf16", 11), _rules(B, R, V, L, "hdrpf", 12)
    rules["length"][:] = torch.tensor([L, L - 3], dtype=torch.int32)
    want = oracle.penalize(_np(x), **{n: _np(v) for n, v in rules.items()})
    _check(ctx.penalize(x, **rules), want, x, "bf16")


@pytest.mark.parametrize("V,L,dtype", [(262144, 131072, "bf16"),        # more different tokens than are counted together
                                       (600011, 9000, "f32")])         # a vocabulary of more than one part
def test_lists_in_several_rounds(ctx, V, L, dtype):
    B, R = 1, 2
    x, rules = _logits(B, R, V, dtype, 21), _rules(B, R, V, 64, "drpfb", 22)
    g = torch.Generator(device="cuda").manual_seed(23)
    rules["history"] = torch.randint(0, V, (B, L), generator=g, device="cuda", dtype=torch.int32)
    rules["length"], rules["prompt_length"] = torch.tensor([L - 1], dtype=torch.int32).cuda(), torch.tensor([L // 3], dtype=torch.int32).cuda()
    want = oracle.penalize(_np(x), **{n: _np(v) for n, v in rules.items()})
    got = ctx.penalize(x, **rules)
    _check(got, want, x, dtype, _changed(rules, B, R, V) | np.isinf(want))
    place = x.clone()
    assert torch.equal(_bits(ctx.penalize(place, **rules, out=place)), _bits(got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_short_and_long_buffers_give_the_same(ctx, dtype):
    # the same history in a buffer that is read by the rows' own CTAs, and in a larger one that a kernel of its own reads
    B, R, V, L = 3, 5, 7001, 900
    x, rules = _logits(B, R, V, dtype, 24), _rules(B, R, V, L, "hdrpfbm", 25)
    long = torch.full((B, 6000), -1, dtype=torch.int32, device="cuda")
    long[:, :L] = rules["history"]
    more = {**rules, "history": long}
    assert torch.equal(_bits(ctx.penalize(x, **rules)), _bits(ctx.penalize(x, **more)))
    assert torch.equal(_bits(ctx.penalize_grad(x, x, **rules)), _bits(ctx.penalize_grad(x, x, **more)))
    a, b = x.clone(), x.clone()
    assert torch.equal(_bits(ctx.penalize(a, **rules, out=a)), _bits(ctx.penalize(b, **more, out=b)))
    # and for a sequence without a token, or with one
    for n in (0, 1):
        rules["length"][:] = n
        rules["prompt_length"][:] = 0
        assert torch.equal(_bits(ctx.penalize(x, **rules)), _bits(ctx.penalize(x, **more)))
    assert ctx.status()[0] == 0


def test_a_wait_that_runs_out_marks_the_rows(ctx):
    x, rules = _logits(8, 4, 30000, "bf16", 26), _rules(8, 4, 30000, 100, "hdrpf", 27)
    want = ctx.penalize(x, **rules)
    ctx.wait_limit(0)
    got = ctx.penalize(x, **rules)
    ctx.wait_limit(2_000_000_000)
    status = ctx.status(clear=True)[0]
    late = got.isnan()
    assert torch.equal(_bits(got)[~late], _bits(want)[~late]) and (status == 8) == bool(late.any())
    assert torch.equal(_bits(ctx.penalize(x, **rules)), _bits(want)) and ctx.status()[0] == 0


def test_two_graphs_and_a_thread_each(ctx):
    # each call has a workspace of its own: two graphs may be replayed side by side, two threads may call at once
    import threading
    sets = [(_logits(3, 3, 20001, "bf16", s), _rules(3, 3, 20001, 5000, "hdrpfb", s)) for s in (31, 32)]
    want = [ctx.penalize(x, **r) for x, r in sets]
    graphs = []
    for x, r in sets:
        out, graph = torch.empty_like(x), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.penalize(x, **r, out=out)
        graphs.append((graph, out))
    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for (graph, out), s in zip(graphs, side):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                out.fill_(7)
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(_bits(out), _bits(w)) for (_, out), w in zip(graphs, want))
    got = [None, None]

    def work(k):
        with torch.cuda.stream(side[k]):
            got[k] = [ctx.penalize(sets[k][0], **sets[k][1]) for _ in range(20)]
            side[k].synchronize()
    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert all(torch.equal(_bits(o), _bits(w)) for outs, w in zip(got, want) for o in outs) and ctx.status()[0] == 0


def test_versions(ctx):
    x, rules = _logits(2, 2, 500, "f32", 33), _rules(2, 2, 500, 20, "hdrpfbm", 34)
    read = [x, *[t for v in rules.values() for t in (v if isinstance(v, tuple) else (v,))]]
    before = [t._version for t in read]
    out = torch.empty_like(x)
    n = out._version
    ctx.penalize(x, **rules, out=out)
    ctx.penalize_grad(x, x, **rules, out=out)
    assert out._version == n + 2 and [t._version for t in read] == before


def test_few_and_many_sequences_give_the_same(ctx):
    B, R, V, L = 400, 2, 20001, 64
    x, rules = _logits(B, R, V, "bf16", 13), _rules(B, R, V, L, "hdrpfbm", 14)
    many = ctx.penalize(x, **rules)
    for b in (0, 1, 2, 399):
        alone = {n: tuple(y[b:b + 1] for y in v) if n == "bias" else v if n == "mask" else v[b:b + 1] for n, v in rules.items()}
        assert torch.equal(_bits(ctx.penalize(x[b:b + 1], **alone)), _bits(many[b:b + 1]))


@pytest.mark.parametrize("law", ["b", "dr", "drpfbm", "hdpf"])
def test_many_sequences_with_short_histories_or_none(ctx, law):
    # so many that the lists are put together beforehand; alone a sequence's rows read what there is themselves
    B, R, V, L = 900, 4, 70001, 30
    x, rules = _logits(B, R, V, "bf16", 41), _rules(B, R, V, L, law, 42)
    many = ctx.penalize(x, **rules)
    grad = ctx.penalize_grad(x, x, **rules)
    for b in (0, 1, 2, 450, 899):
        alone = {n: tuple(y[b:b + 1] for y in v) if n == "bias" else v if n == "mask" else v[b:b + 1] for n, v in rules.items()}
        assert torch.equal(_bits(ctx.penalize(x[b:b + 1], **alone)), _bits(many[b:b + 1]))
        assert torch.equal(_bits(ctx.penalize_grad(x[b:b + 1], x[b:b + 1], **alone)), _bits(grad[b:b + 1]))
    ctx.penalize(x, **rules, out=x)
    assert torch.equal(_bits(x), _bits(many)) and ctx.status()[0] == 0


def test_captured_replayed_and_on_other_streams(ctx):
    B, R, V, L = 6, 4, 30001, 200
    x, rules = _logits(B, R, V, "bf16", 15), _rules(B, R, V, L, "hdrpfbm", 16)
    want = ctx.penalize(x, **rules)
    outs, side = [], [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs += [ctx.penalize(x, **rules) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(_bits(o), _bits(want)) for o in outs)
    out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.penalize(x, **rules, out=out)
    rules["history"].copy_(rules["history"].flip(1))
    rules["length"].clamp_(max=150)
    rules["prompt_length"].clamp_(max=100)
    graph.replay()
    assert torch.equal(_bits(out), _bits(ctx.penalize(x, **rules))) and ctx.status()[0] == 0


def test_autograd(ctx):
    B, R, V, L = 2, 3, 1500, 70
    x, rules = _logits(B, R, V, "f32", 17), _rules(B, R, V, L, "hdrpfbm", 18)
    w = torch.randn((B, R, V), device="cuda")
    leaf = x.clone().requires_grad_(True)
    y = ctx.penalized(leaf, **rules)
    assert torch.equal(_bits(y.detach()), _bits(ctx.penalize(x, **rules)))
    y.backward(w)
    assert torch.equal(leaf.grad, ctx.penalize_grad(w, x, **rules))
    # a gradient that is no tensor of its own (expanded), rules without repetition
    leaf.grad = None
    ctx.penalized(leaf, mask=rules["mask"], mask_row=rules["mask_row"]).sum().backward()
    assert torch.equal(leaf.grad, ctx.penalize_grad(torch.ones_like(x), None, mask=rules["mask"], mask_row=rules["mask_row"]))
    # the history written between the passes
    y = ctx.penalized(leaf, **rules)
    ctx.append(rules["history"], rules["length"] - 5, torch.ones(B, dtype=torch.int32, device="cuda"))
    ctx.status(clear=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(w)
    with pytest.raises(ValueError, match="repetition"):
        ctx.penalized(leaf, **{**rules, "repetition": rules["repetition"].clone().requires_grad_(True)})
    with pytest.raises(ValueError, match="autograd"):
        ctx.penalize(leaf, **rules, out=torch.empty_like(x))
    with pytest.raises(ValueError, match="autograd"):
        ctx.penalize(leaf, **rules)
    with torch.no_grad():
        ctx.penalize(leaf, **rules, out=torch.empty_like(x))
    assert torch.equal(_bits(ctx.penalize(leaf.detach(), **rules)), _bits(ctx.penalize(x, **rules)))


def test_refusals(ps, ctx):
    B, R, V, L = 2, 3, 1000, 40
    x, rules = _logits(B, R, V, "bf16", 19), _rules(B, R, V, L, "hdrpfbm", 20)
    flat = torch.empty(B * R * V + 8, dtype=torch.bfloat16, device="cuda")
    wrong = {
        "history": [rules["history"].long(), rules["history"][:1], rules["history"].t(), rules["history"].cpu(), None],
        "length": [rules["length"].long(), rules["length"][:1], None],
        "prompt_length": [rules["prompt_length"][:1]],
        "draft_tok": [rules["draft_tok"][:, :1], rules["draft_tok"].float()],
        "repetition": [rules["repetition"].double(), rules["repetition"][:1]],
        "presence": [rules["presence"].cpu()],
        "frequency": [rules["frequency"].half()],
        "bias": [rules["bias"][:2], (rules["bias"][0], None, rules["bias"][2]), (rules["bias"][0], rules["bias"][1][:, :3], rules["bias"][2])],
        "mask": [rules["mask"][:, :-1], rules["mask"].long(), rules["mask"][:0], None],
        "mask_row": [rules["mask_row"].long(), rules["mask_row"][:, :1], None],
    }
    for name, values in wrong.items():
        for v in values:
            with pytest.raises((ValueError, ps.PicospecError)):
                ctx.penalize(x, **{**rules, name: v})
    for out in (x.float(), torch.empty((B, R, V + 1), dtype=x.dtype, device="cuda"), flat):
        with pytest.raises(ValueError):
            ctx.penalize(x, **rules, out=out)
    with pytest.raises(ValueError):
        ctx.penalize(x.half(), **rules)
    with pytest.raises(ValueError):
        ctx.penalize_grad(x, None, **rules)                 # repetition needs the logits
    a, b = flat[:B * R * V].view(B, R, V), flat[8:8 + B * R * V].view(B, R, V)
    for call in (lambda: ctx.penalize(a, out=b), lambda: ctx.penalize_grad(a, None, out=b), lambda: ctx.penalize_grad(x, a, **rules, out=a)):
        with pytest.raises(ps.PicospecError) as e:          # overlapping, but not the same place
            call()
        assert e.value.code == ps.binding.EINVAL
    big = torch.zeros((1, 1025), dtype=torch.int32, device="cuda")
    with pytest.raises(ps.PicospecError) as e:
        ctx.penalize(x[:1], bias=(big, big.float(), torch.zeros(1, dtype=torch.int32, device="cuda")))
    assert e.value.code == ps.binding.ECAPACITY
    small = ps.Context(1, 1, V - 1, 1)
    try:
        with pytest.raises(ps.PicospecError) as e:
            small.penalize(x)
        assert e.value.code == ps.binding.ECAPACITY
    finally:
        small.close()
    assert ctx.status()[0] == 0
