"""A call under rules finds what the kernels just before it in the stream have written -- rows, masks, drafted tokens, history, lengths -- and
writes nothing that they still read.  Histories long enough for the list's own kernel, behind which the rows' kernel starts early."""
import pytest
import torch

from oracle import rules as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(1, 1, 1 << 18, 1)
    yield c
    c.close()


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def _set(B, R, V, L, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(hi, *shape):
        return torch.randint(0, hi, shape, generator=g, device="cuda", dtype=torch.int32)
    return dict(x=(4 * torch.randn((B, R, V), generator=g, device="cuda")).to(dtype), history=(ints(V, B, L).double() * torch.rand((B, L), generator=g, device="cuda") ** 3).to(torch.int32),
                length=L - ints(50, B), draft_tok=ints(40, B, R - 1), repetition=1 + torch.rand(B, generator=g, device="cuda"),
                frequency=torch.rand(B, generator=g, device="cuda"), mask=torch.randint(-2 ** 31, 2 ** 31, (3, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int64).to(torch.int32),
                mask_row=ints(4, B, R) - 1)


@pytest.mark.parametrize("B,R,V,L,dtype", [(4, 5, 32001, 9000, torch.bfloat16), (64, 8, 50381, 6000, torch.bfloat16), (3, 3, 128256, 20000, torch.float32)])
def test_what_was_just_written_is_read(ctx, B, R, V, L, dtype):
    sets = [_set(B, R, V, L, dtype, s) for s in (1, 2)]
    want, back = [], []
    for s in sets:
        rules = {n: v for n, v in s.items() if n != "x"}
        want.append(ctx.penalize(s["x"], **rules))
        back.append(ctx.penalize_grad(s["x"], s["x"], **rules))
        torch.cuda.synchronize()
    first = oracle.penalize(**{("logits" if n == "x" else n): v.float().cpu().numpy() if v.is_floating_point() else v.cpu().numpy() for n, v in
                               {k: (v if k in ("mask",) else v[:1]) for k, v in sets[1].items()}.items()})
    torch.testing.assert_close(want[1][:1].double().cpu(), torch.from_numpy(first), rtol=2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24, atol=2.0 ** -40)
    cur = {n: v.clone() for n, v in sets[0].items()}
    rules = {n: v for n, v in cur.items() if n != "x"}
    out, late, seen = torch.empty_like(cur["x"]), torch.empty(64 << 20, device="cuda"), []
    out.copy_(want[0])
    held = want[0]
    for step in range(24):
        s = sets[step % 2]
        if step % 3 == 0:
            late.add_(1.0)              # (so that the host is well ahead of the GPU)
        for n in ("history", "length", "repetition", "frequency", "draft_tok", "mask_row", "mask", "x"):
            cur[n].copy_(s[n])
        if step % 4 == 1:               # in place: the kernel just before reads what the call writes
            source = cur["x"].clone()
            seen.append((ctx.penalize(cur["x"], **rules, out=cur["x"]).clone(), want[step % 2], source, s["x"]))
            continue
        source = out.clone()            # (as does this one)
        if step % 4 == 0:
            ctx.penalize(cur["x"], **rules, out=out)
        else:
            ctx.penalize_grad(cur["x"], cur["x"], **rules, out=out)
        expected = (want if step % 4 == 0 else back)[step % 2]
        seen.append((out.clone(), expected, source, held))
        held = expected
    torch.cuda.synchronize()
    for k, (got, expected, source, before) in enumerate(seen):
        assert torch.equal(_bits(got), _bits(expected)), k
        assert torch.equal(_bits(source), _bits(before)), k
    assert ctx.status()[0] == 0
