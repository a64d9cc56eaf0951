"""A wait that runs out in a call under rules: the pieces of rows concerned are NaN as a whole, all others are right, and the status says so."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SEGMENT = 1024          # a piece of a row is a multiple of so many entries


def _inputs(B, R, V, L, dtype, law, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)
    rules = {}
    if "h" in law:
        rules.update(history=ints(0, V, B, L), length=ints(L // 2, L + 1, B), draft_tok=ints(0, V, B, R - 1),
                     repetition=1 + torch.rand(B, generator=g, device="cuda"), frequency=torch.rand(B, generator=g, device="cuda"))
    if "m" in law:              # every second row has a mask that leaves little
        words = (V + 31) // 32
        rules.update(mask=torch.cat([torch.full((1, words), 0x5F5F5F5F, dtype=torch.int32, device="cuda"), (ints(0, 20, 1, words) == 0).int()]),
                     mask_row=torch.arange(B * R, device="cuda", dtype=torch.int32).view(B, R) % 2)
    return (4 * torch.randn((B, R, V), generator=g, device="cuda")).to(dtype), rules


@pytest.mark.parametrize("law,L", [("", 0), ("m", 0), ("h", 500), ("h", 9000), ("hm", 9000)])
@pytest.mark.parametrize("V,dtype", [(32768, torch.bfloat16), (30001, torch.bfloat16), (30001, torch.float32)])
def test_pieces_are_right_or_nan(V, dtype, law, L):
    import paper_2603_19133_b200 as ps
    ctx = ps.Context(1, 1, V, 1)
    try:
        B, R = 24, 4
        x, rules = _inputs(B, R, V, L, dtype, law, V + L)
        for backward in (False, True):
            def call():
                return ctx.penalize_grad(x, x, **rules) if backward else ctx.penalize(x, **rules)
            want, reached, flush = call(), False, torch.empty(64 << 20, device="cuda")
            for _ in range(20):
                flush.zero_()           # (rows that come from HBM are the later)
                ctx.wait_limit(0)
                got = call()
                ctx.wait_limit(2_000_000_000)
                late = got.isnan()
                assert ctx.status(clear=True)[0] == (8 if bool(late.any()) else 0)
                assert torch.equal(got[~late], want[~late])
                pad = torch.nn.functional.pad(late, (0, -V % SEGMENT), value=False).view(B, R, -1, SEGMENT)
                whole = torch.nn.functional.pad(torch.ones_like(late), (0, -V % SEGMENT), value=False).view(B, R, -1, SEGMENT)
                some = pad.any(-1)
                assert torch.equal(pad[some], whole[some])
                reached |= bool(late.any())
            # without rules the first look comes right behind the copy; else there is work in between, and the copy may have landed by then
            assert reached or law
            assert torch.equal(call(), want) and ctx.status()[0] == 0
    finally:
        ctx.close()
