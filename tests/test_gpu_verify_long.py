"""lg_verify_draft over sequences of more rows than are joined once: the first draft that falls at either
side of that many rows, against 64 bits."""
import math

import pytest
import torch

import q4_ref
from test_gpu_verify import _case, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("m", [65, 66, 130])
def test_the_first_fallen_draft_of_many(cuda, dtype, certain, greedy, m):
    V = 777
    falls = sorted({0, 1, 62, 63, 64, 65, 100, m - 2, m - 1})
    ms = []
    for a in falls:
        ms += [m, 2] if a < m else []
    x, ms, tokens, q, temp, u, r = _case(ms, V, dtype, certain, m)
    temp[:] = 0.0 if greedy else 0.8
    want, t = [], 0
    for b, n in enumerate(ms):
        a = falls[b // 2] if n == m else 1
        for j in range(n - 1):  # drafts stand up to row a: the target's top token, at u = 0
            tokens[t + j + 1] = int(x[t + j].float().argmax())
            u[t + j] = 0.0
        if a < n - 1:           # and a draft that the target never gives
            y = int(x[t + a].float().argmin())
            x[t + a, y] = -math.inf
            tokens[t + a + 1] = y
            if q is not None:
                q[t + a, y] = 0.25
            u[t + a] = 0.5
        want.append(a)
        t += n
    got = _run(cuda, x, ms, tokens, q, temp, u, r)
    assert got[1] == want
    assert got == q4_ref.verify(x, ms, tokens, q, temp, u, r)


def test_a_chunk_of_thousands(cuda):
    """a long chunk scored against its own target: all of it stands but the last row's token"""
    V, m = 100, 3001
    x, ms, tokens, _, _, u, r = _case([m, 1, 64], V, "f32", True, 2)
    tokens[1:m] = x[:m - 1].argmax(-1).int()
    u[:m] = 0.0
    got = _run(cuda, x, ms, tokens, None, None, u, r)
    assert got[1][0] == m - 1
    assert got == q4_ref.verify(x, ms, tokens, None, None, u, r)
