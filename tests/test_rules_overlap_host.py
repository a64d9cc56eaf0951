"""Results that overlap what a call under rules reads are refused, rows that only lie between each other are not.  Without a GPU: on a context that
no device stands behind a call that passes the checks ends with a CUDA error."""
import ctypes
import random

import pytest
import torch

EINVAL, ECUDA = -1, -2
A = 1 << 30


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
    buf[0], buf[1], buf[2], buf[3], buf[4], buf[5] = 0, 1, 1, 100000, 1, 148
    return buf


def _call(lib, fake, p, q, B, R, V, dtype, p_pitch, q_pitch):
    rules = (ctypes.c_char * 256)()
    return lib.picospec_penalize(ctypes.cast(fake, ctypes.c_void_p), p, dtype, B, R, V, p_pitch, ctypes.byref(rules), q, q_pitch, None, None)


def test_rows_between_rows(lib, fake):
    # halves of wider rows, in either order; one element too near, on either side; the same pitch behind the last row
    for dtype, elem in ((0, 4), (1, 2)):
        V, pitch, rows = 1000, 2000, 6
        for apart, code in [(V, ECUDA), (-V, ECUDA), (V - 1, EINVAL), (V + 1, EINVAL), (1 - V, EINVAL), (-1 - V, EINVAL), (V + pitch, ECUDA), (pitch, EINVAL),
                            (5 * pitch, EINVAL), (5 * pitch + V, ECUDA), (5 * pitch + V - 1, EINVAL), (5 * pitch + V + 1, ECUDA), (6 * pitch, ECUDA), (-5 * pitch, EINVAL),
                            (-5 * pitch - V, ECUDA), (-5 * pitch - V + 1, EINVAL), (0, ECUDA)]:
            assert _call(lib, fake, A, A + apart * elem, 2, 3, V, dtype, pitch, pitch) == code, (dtype, apart)
        assert _call(lib, fake, A, A + V * elem, 2, 3, V, dtype, pitch, pitch + 1) == EINVAL
        assert _call(lib, fake, A, A + elem * (5 * pitch + V), 2, 3, V, dtype, pitch, pitch + 1) == ECUDA


def test_rows_as_their_bytes_say(lib, fake):
    g = random.Random(1)
    for _ in range(3000):
        rows, V = g.randint(1, 7), g.randint(1, 9)
        pitch = V + g.choice([0, 0, 1, g.randint(0, 30)])
        apart = g.randint(-rows * pitch - 3, rows * pitch + 3)
        taken = {i * pitch + j for i in range(rows) for j in range(V)}
        meet = apart != 0 and any(i * pitch + j + apart in taken for i in range(rows) for j in range(V))
        assert _call(lib, fake, A, A + 4 * apart, 1, rows, V, 0, pitch, pitch) == (EINVAL if meet else ECUDA), (rows, V, pitch, apart)


def test_the_workspace_is_as_the_header_says(lib):
    # B (V / 256 + 8 min(V, capacity + R + bias_k)) bytes, 12 for the 8 with biases; at most 64 bytes a sequence more
    class Rules(ctypes.Structure):
        _fields_ = [("history", ctypes.c_void_p), ("history_stride", ctypes.c_longlong), ("capacity", ctypes.c_int), ("length", ctypes.c_void_p),
                    ("prompt_length", ctypes.c_void_p), ("draft_tok", ctypes.c_void_p), ("repetition", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                    ("frequency", ctypes.c_void_p), ("bias_idx", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("bias_count", ctypes.c_void_p),
                    ("bias_k", ctypes.c_int), ("mask", ctypes.c_void_p), ("mask_stride", ctypes.c_longlong), ("mask_rows", ctypes.c_int),
                    ("mask_row", ctypes.c_void_p)]
    for B, R, V, capacity, k in [(512, 1, 128256, 131072, 0), (512, 1, 128256, 131072, 300), (64, 8, 151936, 2000, 0), (3, 5, 50381, 7, 11), (1, 1, 1, 1, 0)]:
        r = Rules(history=A, history_stride=capacity, capacity=capacity, length=A, draft_tok=A, repetition=A, bias_idx=A if k else None, bias=A, bias_count=A, bias_k=k)
        said = B * (V / 256 + (12 if k else 8) * min(V, capacity + R + k))
        assert said <= lib.picospec_rules_workspace(ctypes.byref(r), 0, B, R, V) <= said + 64 * B
