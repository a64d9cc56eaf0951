"""Rules, appends and clipping together with the calls they stand beside: drafting, verification and sampling under rules on one history that
stays on the GPU, and a training step of the drafter."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rows
from oracle import rules as rules_oracle

pytestmark = pytest.mark.gpu

B, G, V, K, L = 3, 3, 5003, 24, 64


def _np(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _program(ctx, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"history": torch.randint(0, V, (B, L), generator=g, device="cuda", dtype=torch.int32),
         "prompt": torch.tensor([5, 0, 20], dtype=torch.int32, device="cuda"), "length": torch.tensor([9, 0, 20], dtype=torch.int32, device="cuda"),
         "T": torch.tensor([0.7, 1.0, 1.2], device="cuda"),
         "rules": dict(repetition=torch.tensor([1.3, 1.0, 0.9], device="cuda"), presence=torch.tensor([0.5, 0.0, 1.0], device="cuda"),
                       frequency=torch.tensor([0.2, 0.1, 0.0], device="cuda"),
                       mask=torch.randint(-2 ** 31, 2 ** 31, (4, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int64).to(torch.int32))}
    s["rows"] = torch.randint(-1, 4, (B, G + 1), generator=g, device="cuda", dtype=torch.int32)

    def fresh(step):
        g = torch.Generator(device="cuda").manual_seed(100 * seed + step)
        draft = (3 * torch.randn((B, G, V), generator=g, device="cuda")).to(dtype)
        target = (draft.float().repeat(1, 2, 1)[:, :G + 1] * 0.8 + torch.randn((B, G + 1, V), generator=g, device="cuda")).to(dtype)
        return draft, target, torch.rand((B, G + 1, 3), generator=g, device="cuda").clamp_(max=1 - 2.0 ** -24)
    return s, fresh


def _step(ctx, s, draft, target, u):
    """One draft-and-verify step: the drafter appends what it drafts behind the sequence without counting it, the verifier's outcome is written over it."""
    at, q, drawn, seen = s["length"], [], [], []
    for i in range(G):
        row = ctx.penalize(draft[:, i:i + 1], s["history"], at, s["prompt"], **s["rules"], mask_row=s["rows"][:, i:i + 1].contiguous())
        seen.append(row)
        q.append(ctx.compress(row, s["T"], K, 1.0, K, u[:, i:i + 1, 0].contiguous()))
        drawn.append(q[-1][3])
        at = ctx.append(s["history"], at, drawn[-1][:, 0].contiguous())
    tok = torch.cat(drawn, 1)
    idx, prob, count = (torch.cat([x[k] for x in q], 1) for k in range(3))
    under = ctx.penalize(target, s["history"], s["length"], s["prompt"], tok, **s["rules"], mask_row=s["rows"], out=target)
    out = ctx.verify(under, s["T"], tok, idx, prob, count, u[:, :G, 1].contiguous(), u[:, G, 1:].contiguous())
    ctx.append(s["history"], s["length"], out["token"], tok, out["accept_len"], out=s["length"])
    return {"rows": torch.cat(seen, 1), "tok": tok, "idx": idx, "prob": prob, "count": count, "under": under, **out}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_on_a_history_that_stays_on_the_gpu(dtype):
    import paper_2603_19133_b200 as ps
    ctx = ps.Context(B, G, V, K)
    rtol = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    try:
        s, fresh = _program(ctx, dtype, 1)
        fixed = {n: _np(v) for n, v in s["rules"].items()}
        for step in range(4):
            draft, target, u = fresh(step)
            raw, before, length = _np(target), _np(s["history"]), _np(s["length"])
            o = _step(ctx, s, draft, target, u)
            # the rows under rules, against the statement (double precision rounded once; terms below 2^7)
            for i in range(G):
                seen = before.copy()
                for b in range(B):
                    seen[b, length[b]:length[b] + i] = _np(o["tok"])[b, :i]
                want = rules_oracle.penalize(_np(draft[:, i:i + 1]), seen, length + i, _np(s["prompt"]), **fixed, mask_row=_np(s["rows"])[:, i:i + 1])
                np.testing.assert_allclose(_np(o["rows"])[:, i:i + 1], want, rtol=rtol, atol=2.0 ** -43)
            want = rules_oracle.penalize(raw, before, length, _np(s["prompt"]), _np(o["tok"]), **fixed, mask_row=_np(s["rows"]))
            np.testing.assert_allclose(_np(o["under"]), want, rtol=rtol, atol=2.0 ** -43)
            # what was verified, and where it went
            v = oracle.verify(_np(o["under"]), _np(s["T"]), _np(o["tok"]), _np(o["idx"]), _np(o["prob"]), _np(o["count"]), _np(u[:, :G, 1]), _np(u[:, G, 1:]),
                              nthreads=oracle.cores())
            assert np.array_equal(_np(o["accept_len"]), v["accept_len"]) and np.array_equal(_np(o["token"]), v["token"])
            history, after, bad = rules_oracle.append(before, length, v["token"], _np(o["tok"]), v["accept_len"])
            assert not bad and np.array_equal(_np(s["length"]), after)
            for b in range(B):
                assert np.array_equal(_np(s["history"])[b, :after[b]], history[b, :after[b]])
        # a token without a drafter
        draft, _, u = fresh(9)
        row = ctx.penalize(draft[:, :1], s["history"], s["length"], s["prompt"], **s["rules"], mask_row=s["rows"][:, :1].contiguous())
        token = ctx.sample(row, s["T"], u[:, :1, :2].contiguous())[0]
        assert np.array_equal(_np(token), rows.sample(_np(row), _np(s["T"]), _np(u[:, :1, :2]))[0])
        length = s["length"].clone()
        ctx.append(s["history"], s["length"], token[:, 0].contiguous(), out=s["length"])
        assert torch.equal(s["length"], length + 1) and all(int(s["history"][b, length[b]]) == int(token[b, 0]) for b in range(B))
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_steps_in_one_graph():
    import paper_2603_19133_b200 as ps
    ctx = ps.Context(B, G, V, K)
    try:
        eager, fresh = _program(ctx, torch.bfloat16, 2)
        replayed, _ = _program(ctx, torch.bfloat16, 2)
        draft, target, u = fresh(0)
        scratch, _ = _program(ctx, torch.bfloat16, 2)
        _step(ctx, scratch, draft.clone(), target.clone(), u)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = _step(ctx, replayed, draft, target, u)
        for step in range(3):
            new = fresh(step)
            for x, y in zip((draft, target, u), new):
                x.copy_(y)
            graph.replay()
            o = _step(ctx, eager, *new)
            assert all(torch.equal(captured[n], o[n]) for n in ("tok", "accept_len", "token", "count"))
            assert torch.equal(replayed["history"], eager["history"]) and torch.equal(replayed["length"], eager["length"])
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_a_training_step_under_rules():
    # a drafter of one embedding and one head, trained on teacher rows that were taken under rules
    import paper_2603_19133_b200 as ps
    R, D = 4, 32
    g = torch.Generator(device="cuda").manual_seed(5)
    ctx = ps.Context(B, R, V, K)
    try:
        tokens = torch.randint(0, V, (B, R), generator=g, device="cuda", dtype=torch.int32)
        rules = dict(history=torch.randint(0, V, (B, L), generator=g, device="cuda", dtype=torch.int32), length=torch.full((B,), L, dtype=torch.int32, device="cuda"),
                     draft_tok=tokens[:, 1:].contiguous(), repetition=torch.tensor([1.2, 1.0, 1.4], device="cuda"), presence=torch.full((B,), 0.3, device="cuda"),
                     mask=torch.full((1, (V + 31) // 32), 0x5F5F5F5F, dtype=torch.int32, device="cuda"), mask_row=torch.zeros((B, R), dtype=torch.int32, device="cuda"))
        T = torch.ones(B, device="cuda")
        teacher = ctx.penalize(3 * torch.randn((B, R, V), generator=g, device="cuda"), **rules)
        t_idx, t_prob, t_count, _ = ctx.compress(teacher, T, K, 1.0, K)
        emb = (0.3 * torch.randn((V, D), generator=g, device="cuda")).requires_grad_(True)
        head = (0.3 * torch.randn((V, D), generator=g, device="cuda")).requires_grad_(True)
        loss = ctx.distill_loss(ctx.penalized(emb[tokens.long()] @ head.T, **rules), T, t_idx, t_prob, t_count).mean()
        loss.backward()
        grads = [emb.grad.clone(), head.grad.clone()]

        # the same in double precision with plain operations
        e64, h64 = emb.detach().double().requires_grad_(True), head.detach().double().requires_grad_(True)
        x = e64[tokens.long()] @ h64.T
        made = torch.zeros((B, R, V), dtype=torch.bool, device="cuda")
        for b in range(B):
            for i in range(R):
                made[b, i, rules["history"][b].long()] = True
                made[b, i, rules["draft_tok"][b, :i].long()] = True
        rho = rules["repetition"].double()[:, None, None]
        y = torch.where(made, torch.where(x > 0, x / rho, x * rho), x) - 0.3 * made      # (0.3 in fp32 against 0.3: a constant, no gradient)
        v = torch.arange(V, device="cuda")
        allowed = (0x5F5F5F5F >> (v % 32)) & 1 != 0
        y = y.masked_fill(~allowed, -float("inf"))
        log_s = torch.log_softmax(y, -1).gather(-1, t_idx.clamp(min=0).long())
        t = t_prob.double()
        want = torch.where(t > 0, t * (t.clamp(min=1e-300).log() - log_s), 0.0).sum(-1).mean()
        want.backward()
        # (losses to the sums' 6.6e-6; gradients: the row's coefficients to 7e-6 of its largest, then products over V or B R terms in fp32)
        np.testing.assert_allclose(float(loss.detach()), float(want.detach()), rtol=2.0 ** -20, atol=6.6e-6)
        for a, b in zip(grads, (e64.grad, h64.grad)):
            assert float((a.double() - b).norm()) <= 4e-5 * float(b.norm())

        # clipped as plain operations clip
        norm = ctx.clip_grad([emb.grad, head.grad], 1e-3)
        whole = torch.cat([x.double().flatten() for x in grads]).norm()
        np.testing.assert_allclose(float(norm), float(whole), rtol=34 * 2.0 ** -24)
        scale = min(1.0, float(np.float32(1e-3)) / float(whole))
        for a, b in zip((emb.grad, head.grad), grads):
            np.testing.assert_allclose(_np(a), _np(b).astype(np.float64) * scale, rtol=36 * 2.0 ** -24, atol=2.0 ** -149)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()


def test_the_kernels_are_bracketed_when_profiling():
    import paper_2603_19133_b200 as ps
    ctx = ps.Context(1, 1, V, 1)
    try:
        ctx.profile_enable(1)
        x, n = torch.randn((2, 2, V), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        history = torch.zeros((2, 9000), dtype=torch.int32, device="cuda")
        for _ in range(3):
            ctx.penalize(x, history, n, repetition=torch.ones(2, device="cuda"))
            ctx.append(history, n, n)
            ctx.clip_grad([x], 1.0)
        for kind in (9, 10, 11, 12):
            ms = ctx.profile_samples(kind)
            assert len(ms) == 3 and all(t > 0 for t in ms)
        ctx.profile_enable(0)
    finally:
        ctx.close()
