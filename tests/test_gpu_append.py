"""Tokens put behind a history, exactly, against the statement in oracle/rules.py."""
import numpy as np
import pytest
import torch

from oracle import rules as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    import paper_2603_19133_b200 as ps
    c = ps.Context(1, 1, 1000, 1)
    yield c
    c.close()


def _np(t):
    return None if t is None else t.cpu().numpy()


def _inputs(B, G, L, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)

    draft = ints(0, 1000, B, G) if G else None
    accept = ints(-1, G + 1, B) if G else None
    return ints(0, 1000, B, L), ints(0, max(1, L - G), B), ints(0, 1000, B), draft, accept


@pytest.mark.parametrize("B,G,L,pad", [(1, 0, 1, 0), (1, 4, 100, 0), (7, 1, 10, 3), (9, 8, 64, 0), (300, 16, 500, 5), (3, 100, 1000, 0)])
@pytest.mark.parametrize("last", [True, False])
def test_append(ctx, B, G, L, pad, last):
    history, length, token, draft, accept = _inputs(B, G, L, B + G)
    if not last and G == 0:
        return
    buf = torch.full((B, L + pad), -5, dtype=torch.int32, device="cuda")
    buf[:, :L] = history
    token = token if last else None
    want, want_length, bad = oracle.append(_np(history), _np(length), _np(token), _np(draft), _np(accept))
    got = ctx.append(buf[:, :L], length, token, draft, accept)
    assert np.array_equal(_np(buf[:, :L]), want) and np.array_equal(_np(got), want_length) and bool((buf[:, L:] == -5).all())
    assert ctx.status(clear=True)[0] == (4 if bad else 0)
    # in place of the lengths
    buf[:, :L] = history
    assert ctx.append(buf[:, :L], length, token, draft, accept, out=length) is length
    assert np.array_equal(_np(buf[:, :L]), want) and np.array_equal(_np(length), want_length)


def test_sequences_with_bad_data_are_left_alone(ctx):
    B, G, L = 9, 4, 20
    history, length, token, draft, accept = _inputs(B, G, L, 1)
    accept[:], length[:] = 2, 5
    accept[0] = G + 1
    accept[1] = -2                      # not decided yet: no fault
    length[2] = -1
    length[3] = L + 1
    length[4] = L - 2                   # room for two of three
    length[5] = L - 3                   # just room
    draft[6, 1] = -1
    draft[7, 2] = -1                    # behind what was accepted
    token[8] = -1
    want, want_length, bad = oracle.append(_np(history), _np(length), _np(token), _np(draft), _np(accept))
    assert bad and (want_length != _np(length)).tolist() == [False, False, False, False, False, True, False, True, False]
    rest = torch.cat([history, torch.full((3, L), 7, dtype=torch.int32, device="cuda")])
    got = ctx.append(rest[:B], length, token, draft, accept)
    assert np.array_equal(_np(rest[:B]), want) and np.array_equal(_np(got), want_length) and bool((rest[B:] == 7).all())
    assert ctx.status(clear=True)[0] == 4
    accept[:] = -1
    assert torch.equal(ctx.append(rest[:B], length, token, draft, accept), length) and ctx.status()[0] == 0


def test_offsets_beyond_32_bits(ctx):
    pitch = 1 << 30
    history = torch.empty(2 * pitch + 50, dtype=torch.int32, device="cuda").as_strided((3, 50), (pitch, 1))
    history.zero_()
    token = torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda")
    length = ctx.append(history, torch.tensor([0, 49, 3], dtype=torch.int32, device="cuda"), token)
    assert length.tolist() == [1, 50, 4] and [int(history[0, 0]), int(history[1, 49]), int(history[2, 3])] == [5, 6, 7]


def test_captured_and_replayed(ctx):
    history, length, token, draft, accept = _inputs(5, 3, 200, 2)
    accept.clamp_(min=0)
    length[:] = 10
    ctx.append(history, length, token, draft, accept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.append(history, length, token, draft, accept, out=length)
    want, want_length = _np(history), _np(length)
    for _ in range(3):
        graph.replay()
        want, want_length, _ = oracle.append(want, want_length, _np(token), _np(draft), _np(accept))
    assert np.array_equal(_np(history), want) and np.array_equal(_np(length), want_length) and ctx.status()[0] == 0


def test_refusals(ctx):
    import paper_2603_19133_b200 as ps
    history, length, token, draft, accept = _inputs(4, 3, 50, 3)
    for args in [(history.long(), length, token, draft, accept), (history, length.long(), token, draft, accept), (history, length, None, None, None),
                 (history, length, token, draft, None), (history, length, token, None, accept), (history, length[:2], token, draft, accept),
                 (history.t(), length, token, draft, accept), (history[0].expand(4, -1), length, token, draft, accept),
                 (history.cpu(), length, token, draft, accept), (None, length, token, draft, accept), (history, length, token[:2], draft, accept)]:
        with pytest.raises((ValueError, ps.PicospecError)):
            ctx.append(*args)
    assert ctx.append(history[:0], length[:0], token[:0]).shape == (0,)
    assert ctx.status()[0] == 0
