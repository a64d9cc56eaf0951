"""The ways a row can take through the sampling kernel, with clusters of several CTAs and more rows than run at a time: CTAs end at
different times and others take their places on the SM."""
import pytest
import torch

from test_gpu_sample import _check, _stored, _uniforms, _zipf, ps  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,V", [("bf16", 140001), ("f32", 70001)])
def test_min_p_alone_in_many_rows(ps, dtype, V):
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = _stored(_zipf(160, 2, V, g), dtype)
    T = 0.4 + torch.rand((160,), generator=g, device="cuda")
    _check(ps, logits, T, _uniforms(160, 2, g), None, None, 1e-3 + torch.rand((160,), generator=g, device="cuda") ** 3)


def test_entries_of_a_bin_put_in_order_in_many_rows(ps):
    g = torch.Generator(device="cuda").manual_seed(43)
    V = 70001
    logits = _stored(_zipf(160, 2, V, g), "f32")
    T = 0.4 + torch.rand((160,), generator=g, device="cuda")
    k = torch.randint(1, 1200, (160,), generator=g, device="cuda", dtype=torch.int32)
    p = 0.3 + 0.69 * torch.rand((160,), generator=g, device="cuda")
    _check(ps, logits, T, _uniforms(160, 2, g), k)
    _check(ps, logits, T, _uniforms(160, 2, g), None, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_draws_on_borders_of_chunks_in_many_rows(ps, dtype):
    # no limits; 64 chunks of the same mass: a uniform of j / 64 lies on a border, so every row takes its exact sums
    g = torch.Generator(device="cuda").manual_seed(47)
    V, n = 65536, 400
    logits = _stored(torch.full((1, 1, 1), 0.5, device="cuda").expand(n, 1, V), dtype)
    u = _uniforms(n, 1, g)
    u[:, 0, 0] = torch.randint(0, 64, (n,), generator=g, device="cuda") / 64.0
    got, slow = _check(ps, logits, torch.ones(n, device="cuda"), u)
    assert slow == int((u[:, 0, 0] > 0).sum())
    assert torch.equal(got[0][:, 0] // 1024, (u[:, 0, 0] * 64).to(torch.int32))
