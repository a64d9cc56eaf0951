"""Calls on dense rows may overlap on one context; with the per-kernel timing on as well."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

SAMPLE, DISTILL = 7, 8          # PICOSPEC_PROF_SAMPLE, PICOSPEC_PROF_DISTILL


def test_launches_of_several_threads_are_each_recorded():
    import paper_2603_19133_b200 as ps
    V, K, N = 5000, 4, 30
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((2, 1, V), generator=g, device="cuda")
    T, u = torch.ones(2, device="cuda"), torch.rand((2, 1, 2), generator=g, device="cuda")
    idx = torch.arange(K, dtype=torch.int32, device="cuda").expand(2, 1, K).contiguous()
    t, n = torch.full((2, 1, K), 0.25, device="cuda"), torch.full((2, 1), K, dtype=torch.int32, device="cuda")
    ctx = ps.Context(1, 1, V, K)
    failed = []
    try:
        ctx.sample(x, T, u), ctx.distill(x, T, idx, t, n)
        ctx.profile_enable(1)
        start = threading.Barrier(4)

        def work():
            try:
                start.wait()
                with torch.cuda.stream(torch.cuda.Stream()):
                    for _ in range(N):
                        ctx.sample(x, T, u)
                        ctx.distill(x, T, idx, t, n)
                torch.cuda.synchronize()
            except Exception as e:      # (reported by the test's own thread)
                failed.append(e)

        for _ in range(5):
            torch.cuda.synchronize()
            threads = [threading.Thread(target=work) for _ in range(4)]
            [th.start() for th in threads]
            [th.join() for th in threads]
            assert not failed
            for kind in (SAMPLE, DISTILL):
                ms = ctx.profile_samples(kind)
                # (between one thread's events only its own launch may lie)
                assert len(ms) == 4 * N and all(0 < m < 5 for m in ms)
        ctx.profile_enable(0)
        assert ctx.status()[0] == 0
    finally:
        ctx.close()
