"""lg_verify_draft at r = 0: the first token that has mass, without a second search of the row where no
draft's probabilities are taken off it."""
import math

import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg
from test_gpu_verify import _case, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("r", [0.0, -1.0, math.nan, 2.0 ** -149])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("batch", [1, 30, 170])
def test_the_first_mass(cuda, batch, certain, r):
    """the first tokens masked, or some 2^-45 of the mass each; with a draft's row what it leaves"""
    V = 5000
    x, ms, tokens, q, _, u, _ = _case([2] * batch, V, "f32", certain, batch)
    x[:, :70] = -math.inf
    x[0::4, 70:200] = x[0::4].amax(-1, keepdim=True) - 31.0
    u[0::2] = 1 - 2.0 ** -24
    c = (x, ms, tokens, q, None, u, torch.full((batch,), r))
    assert _run(cuda, *c) == q4_ref.verify(*c)


def test_zero_costs_no_second_search(cuda):
    """64 sequences whose numbers are all zero against numbers in the middle of tokens: the second search
    takes several times a call (best of 20 each)"""
    V, batch = 64000, 64
    x = (torch.randn((batch, V), generator=torch.Generator().manual_seed(3)) * 2).bfloat16().to(cuda)
    ch = lg.Chunk.of([1] * batch, cuda)
    tokens = torch.zeros(batch, dtype=torch.int32, device=cuda)
    picked, accepted, status = (torch.zeros(n, dtype=torch.int32, device=cuda) for n in (batch, batch, 1))
    ws = torch.empty(lg.lg_verify_workspace_size(x, ch), dtype=torch.uint8, device=cuda)
    u = torch.full((batch,), 0.5, device=cuda)
    x[:, 0] = x.amax() + 4.0  # a large part of the line: its middle is next to no bound
    middle = (x.cpu().double().softmax(-1)[:, 0] / 2).float().to(cuda)
    assert float(middle.min()) > 2.0 ** -20

    def best(r):
        times = []
        for _ in range(20):
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            e[0].record()
            for _ in range(5):
                lg.lg_verify_draft(x, ch, tokens, None, None, u, r, picked, accepted, ws, status)
            e[1].record()
            torch.cuda.synchronize()
            times.append(e[0].elapsed_time(e[1]))
        assert picked.tolist() == [0] * batch
        return min(times)

    assert best(torch.zeros(batch, device=cuda)) < 1.5 * best(middle)
