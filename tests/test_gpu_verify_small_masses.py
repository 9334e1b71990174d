"""lg_verify_draft where little is left of a row after its draft: the next token is written whatever the
masses are, from what is left where that reaches 2^-60 of the mass an element, else from the row itself."""
import math

import pytest
import torch

from test_gpu_verify import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [1, 7, 170])  # clusters of sixteen CTAs to one
@pytest.mark.parametrize("bits", [40, 55, 59, 59.5, 60, 61, 61.5, 62, 62.5, 63, 63.5, 64, 65, 66, 67, 75])
def test_a_token_is_written_whatever_is_left(cuda, dtype, batch, bits):
    """one token holds all but the others' 2^-bits each, and the draft claims it whole; the drafted token
    is another one that falls, since the draft gives it more than u times its mass"""
    V, top, y, m = 1000, 137, 5, 2 * batch
    temp = 1.0 if dtype == "f32" else 0.25  # (bf16 steps of a logit of 11 are 2^-4)
    x = torch.full((m, V), -bits * math.log(2) * temp)
    x[:, top] = 0.0
    x = x if dtype == "f32" else x.bfloat16()
    mass = math.exp(float(x[0, 0]) / temp) * 2.0 ** 62  # of one of the others, in 2^-62
    q = torch.zeros((m, V))
    q[:, top], q[:, y] = 1.0, 2.0 ** -20
    gen = torch.Generator().manual_seed(1)
    at = torch.randint(0, V - 2, (batch,), generator=gen)  # of the tokens that keep their mass
    r = ((at.double() + 0.5) / (V - 2)).float()
    picked, accepted = _run(cuda, x, [2] * batch, torch.full((m,), y, dtype=torch.int32), q,
                            torch.full((batch,), temp), torch.full((m,), 0.5), r)
    assert accepted == [0] * batch
    assert picked[1::2] == [-1] * batch
    left = [i for i in range(V) if i not in (top, y)]
    for b in range(batch):
        if mass >= 4.0:      # 2^-60
            assert picked[2 * b] == left[int(at[b])]
        elif mass < 0.99:    # nothing is left to 2^-62: the row itself, whose mass is the top token's
            assert picked[2 * b] == top
        else:
            assert picked[2 * b] in (top, left[int(at[b])])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masses_next_to_the_least(cuda, dtype):
    """32 tokens of 2^-55 in one part of the row, and everywhere else 2^-63.5, which together are more but
    count as zero each: the next token is one of the 32, all alike"""
    V, top, y, batch = 40000, 39000, 5, 8
    m, temp = 2 * batch, 0.25
    x = torch.full((m, V), -63.5 * math.log(2) * temp)
    few = list(range(20000, 20032))
    x[:, few] = -55 * math.log(2) * temp
    x[:, top] = 0.0
    x = x if dtype == "f32" else x.bfloat16()
    q = torch.zeros((m, V))
    q[:, top], q[:, y] = 1.0, 2.0 ** -20
    at = torch.arange(batch) * 4
    r = ((at.double() + 0.5) / 32).float()
    picked, accepted = _run(cuda, x, [2] * batch, torch.full((m,), y, dtype=torch.int32), q,
                            torch.full((batch,), temp), torch.full((m,), 0.5), r)
    assert accepted == [0] * batch
    assert picked[0::2] == [few[i] for i in at]
