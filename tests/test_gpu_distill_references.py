"""Distillation where a warp moves its running sum from one reference to another and the references lie beyond fp32's reach in units of the
temperature: two masks of different large values, large logits, a tiny temperature."""
import pytest
import torch

from test_gpu_distill import _check, ps  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

ROWS, V, K = 80, 20480, 9       # a CTA a row: each of its warps takes chunks c, c + 8 and c + 16


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("values", ["two_masks", "near_masks", "large", "tiny_temperature", "rising"])
def test_references_beyond_reach(ps, values, dtype, tail):
    g = torch.Generator(device="cuda").manual_seed(83)
    x = torch.randn((1, ROWS, V), generator=g, device="cuda") * 2
    chunk = x.view(1, ROWS, V // 1024, 1024)
    lowest, T = torch.finfo(dtype).min, 0.3
    masked = torch.zeros(V // 1024, dtype=torch.bool)
    if values == "two_masks":               # the type's lowest value, then another one, then ordinary chunks
        chunk[:, :, 0], chunk[:, :, 8] = lowest, -1e38
        chunk[:, :, 1], chunk[:, :, 9], chunk[:, :, 17] = lowest, -2e38, -1.5e38      # (a warp that sees nothing else)
        masked[[0, 8, 1, 9, 17]] = True
    elif values == "near_masks":            # fp32's lowest and bf16's
        chunk[:, :, 2], chunk[:, :, 10] = lowest, torch.finfo(torch.bfloat16).min * (1 - 2.0 ** -7)
        chunk[:, :, 3], chunk[:, :, 11] = lowest, torch.finfo(torch.bfloat16).min
        masked[[2, 10, 3, 11]] = True
    elif values == "large":                 # positive, growing by chunk: beyond reach from the first
        x.mul_(1e36)
        chunk += 2e38 + 5e36 * torch.arange(V // 1024, device="cuda")[:, None]
    elif values == "tiny_temperature":
        T = 1e-37
        chunk += 25 + torch.arange(V // 1024, device="cuda")[:, None] / 4
    else:                                   # from within reach to beyond it
        T = 1e-8
        chunk += 0.5 * torch.arange(V // 1024, device="cuda")[:, None] ** 2
    logits = x.to(dtype)
    allowed = torch.arange(V, device="cuda")[~masked.cuda().repeat_interleave(1024)]
    pick = torch.rand((1, ROWS, allowed.numel()), generator=g, device="cuda").topk(K, -1).indices
    idx = allowed[pick].to(torch.int32).contiguous()
    if values == "large":                   # (the loss of any other entry is beyond fp32)
        idx[:, :, 0] = logits.argmax(-1).to(torch.int32)
        idx[:, :, 1:] = torch.arange(1, K, dtype=torch.int32, device="cuda")
    t = torch.rand((1, ROWS, K), generator=g, device="cuda")
    t = t / t.sum(-1, keepdim=True) * 0.9
    if values == "large":
        t[:, :, 1:] = 0.0
    count = torch.full((1, ROWS), K, dtype=torch.int32, device="cuda")
    temperature = torch.tensor([T], device="cuda")
    weight = torch.rand((1, ROWS), generator=g, device="cuda") * min(1.0, T * 1e30)
    ctx = ps.Context(1, 1, V, K)
    try:
        got = ctx.distill(logits, temperature, idx, t, count, weight=weight, tail=tail)
        assert ctx.status(clear=True)[0] == 0
        _check(got, logits, temperature, idx, t, count, weight, tail)
        few = [v[:, :2].contiguous() for v in (logits, idx, t, count, weight)]      # a row in several CTAs
        got = ctx.distill(few[0], temperature, *few[1:4], weight=few[4], tail=tail)
        _check(got, few[0], temperature, *few[1:], tail)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()
