"""The calls around a step: what they record, allocate, hold on to and refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(1, 1, 200000, 1)
    yield c
    c.close()


def test_a_norm_is_recorded_as_a_norm(ctx):
    # 11: grad_norm, and clip_grad's pass over the squares; 12: the pass that scales, which grad_norm has none of
    g = torch.randn(5000, device="cuda")
    ctx.profile_enable(1)
    for _ in range(3):
        ctx.grad_norm([g])
    assert len(ctx.profile_samples(11)) == 3 and len(ctx.profile_samples(12)) == 0
    norm = ctx.grad_norm([g])
    for _ in range(2):
        ctx.clip_grad([g], 1.0)
    ctx.clip_grad([g], 1.0, norm=norm)
    assert len(ctx.profile_samples(11)) == 3 and len(ctx.profile_samples(12)) == 3
    ctx.profile_enable(0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [4096, 50381])
def test_rows_far_apart_give_rows_that_are_not(ctx, dtype, V):
    # the last positions of a model's output: their pitch is the text's length times the vocabulary
    B, S = 3, 40
    output = torch.randn((B, S, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    last = output[:, -1:]
    rules = dict(history=torch.randint(0, V, (B, 100), device="cuda", dtype=torch.int32), length=torch.full((B,), 100, dtype=torch.int32, device="cuda"),
                 repetition=torch.full((B,), 1.5, device="cuda"))
    want = ctx.penalize(last.contiguous(), **rules)
    leaf = output.clone().requires_grad_(True)
    for got in (ctx.penalize(last, **rules), ctx.penalize_grad(last, last, **rules), ctx.penalized(leaf[:, -1:], **rules).detach()):
        assert got.shape == last.shape and got.stride(2) == 1
        assert got.untyped_storage().nbytes() <= B * (V * got.element_size() + 16)
        # rows on 16-byte boundaries stay on them, and others as far from them as they were
        assert (got.stride(0) - last.stride(0)) * got.element_size() % 16 == 0
    assert torch.equal(ctx.penalize(last, **rules), want) and torch.equal(ctx.penalized(leaf[:, -1:], **rules).detach(), want)
    assert torch.equal(ctx.penalize_grad(last, last, **rules), ctx.penalize_grad(last.contiguous(), last.contiguous(), **rules))
    # a few elements of padding
    flat = torch.empty(B * (V + 5), dtype=dtype, device="cuda")
    padded = flat.view(B, 1, V + 5)[..., :V].copy_(last)
    assert torch.equal(ctx.penalize(padded, **rules), want)
    assert ctx.status()[0] == 0


def test_a_list_of_gradients_that_another_thread_changes(ctx):
    # the call lets other threads run while it launches: what it was given stays alive, whatever becomes of the list
    import sys
    import threading
    live = [torch.ones(1000 + i, device="cuda") for i in range(300)]
    stop = threading.Event()

    def change():
        k = 0
        while not stop.is_set():
            k += 1
            if k % 2:
                live.clear()
            live[:] = [torch.ones(1000 + i, device="cuda") for i in range(300)]
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    worker = threading.Thread(target=change)
    worker.start()
    try:
        for _ in range(150):
            ctx.clip_grad(live, 1.0)
            ctx.grad_norm(live)
    finally:
        stop.set()
        worker.join()
        sys.setswitchinterval(interval)
    # and nothing is kept: the references are given back, also where the call is refused
    g = torch.ones(10, device="cuda")
    bad = torch.ones(10, device="cuda", dtype=torch.float64)
    lists = ([g, None], (g,), [g, bad])
    before = [sys.getrefcount(x) for x in (g, bad, *lists)], torch._C._storage_Use_Count(g.untyped_storage()._cdata)
    for _ in range(20):
        ctx.grad_norm(lists[0])
        ctx.clip_grad(lists[1], 1.0)
        with pytest.raises(ValueError):
            ctx.clip_grad(lists[2], 1.0)
    assert ([sys.getrefcount(x) for x in (g, bad, *lists)], torch._C._storage_Use_Count(g.untyped_storage()._cdata)) == before
    assert ctx.status()[0] == 0


def test_a_norm_that_lies_in_what_is_written_is_refused(ctx):
    # every part of the pass that scales reads it, at no time in particular
    flat = torch.full((64,), 3.0, device="cuda")
    grads, half = [flat[:10], flat[16:40]], torch.ones(8, device="cuda").to(torch.bfloat16)
    for norm in (flat[0:1], flat[9:10], flat[39:40]):
        with pytest.raises(ValueError, match="norm lies in"):
            ctx.clip_grad(grads, 1.0, norm=norm)
    with pytest.raises(ValueError, match="norm lies in"):
        ctx.clip_grad([half], 1.0, norm=half.view(torch.float32)[3:])
    out = [torch.empty_like(g) for g in grads]
    with pytest.raises(ValueError, match="norm lies in"):
        ctx.clip_grad(grads, 1.0, norm=out[1][:1], out=out)
    assert bool((flat == 3).all())
    # beside them, or in what is read alone, it may
    for norm in (flat[10:11], flat[15:16], flat[40:41]):
        ctx.clip_grad(grads, 30.0, norm=norm)
    ctx.clip_grad(grads, 1.0, norm=flat[0:1], out=out)
    assert bool((flat == 3).all()) and all(bool(((o - 1).abs() <= 2.0 ** -22).all()) for o in out)
    assert ctx.status()[0] == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [5003, 8192])
@pytest.mark.parametrize("L", [100, 9000])
def test_results_between_the_rows_that_are_read(ctx, dtype, V, L):
    B, R = 3, 4
    g = torch.Generator(device="cuda").manual_seed(V + L)
    wide = torch.randn((B, R, 2, V), device="cuda", generator=g).to(dtype)
    x, out = wide[:, :, 0], wide[:, :, 1]
    rules = dict(history=torch.randint(0, V, (B, L), device="cuda", dtype=torch.int32, generator=g), length=torch.full((B,), L, dtype=torch.int32, device="cuda"),
                 draft_tok=torch.randint(0, V, (B, R - 1), device="cuda", dtype=torch.int32, generator=g), repetition=torch.full((B,), 1.5, device="cuda"),
                 mask=torch.randint(-2 ** 31, 2 ** 31, (2, (V + 31) // 32), device="cuda", dtype=torch.int64, generator=g).to(torch.int32),
                 mask_row=torch.randint(-1, 2, (B, R), device="cuda", dtype=torch.int32, generator=g))
    before = x.clone()
    want, back = ctx.penalize(before, **rules), ctx.penalize_grad(before, before, **rules)
    assert ctx.penalize(x, **rules, out=out) is out
    assert torch.equal(out, want) and torch.equal(x, before)
    ctx.penalize_grad(x, x, **rules, out=out)
    assert torch.equal(out, back) and torch.equal(x, before) and ctx.status()[0] == 0


@pytest.mark.parametrize("L", [200, 9000])
def test_a_training_step_under_rules_in_one_graph(ctx, L):
    # forward, backward and clipping captured together and replayed on new rows, histories and penalties
    B, R, V = 3, 4, 5003
    g = torch.Generator(device="cuda").manual_seed(L)
    head = torch.randn((B, R, V), device="cuda", generator=g).requires_grad_(True)
    x, w = (torch.randn((B, R, V), device="cuda", generator=g) for _ in range(2))
    history = torch.randint(0, V, (B, L), device="cuda", dtype=torch.int32, generator=g)
    length, rho = torch.full((B,), L // 2, dtype=torch.int32, device="cuda"), torch.full((B,), 1.25, device="cuda")

    def step():
        y = ctx.penalized(x * head, history, length, repetition=rho, frequency=rho)
        grad, = torch.autograd.grad((y * w).sum(), head)
        return grad, ctx.clip_grad([grad], 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        x.normal_(generator=g)
        history.copy_(history.roll(k + 1, 1).flip(0))
        length.add_(7)
        rho.mul_(1.1)
        graph.replay()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and float(want[0].norm()) > 0.99
    assert ctx.status()[0] == 0
