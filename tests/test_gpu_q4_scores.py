"""Scores over a 4-bit cache carry the precision of fp32, also where a group's least value is large beside its
range: the largest score of single tokens against 64 bits."""
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,g", [(64, 7), (128, 4)])
@pytest.mark.parametrize("batch,n", [(2, 300), (2, 7000), (90, 200)])  # clusters, and lines
@pytest.mark.parametrize("mean", [0.0, 20.0, -300.0])
def test_the_largest_score(cuda, d, g, batch, n, mean):
    """Products of codes and queries are exact, and so are those of least values with the groups' sums of q
    (an fp32 number in three bf16 terms).  What rounds: a group's sum of q, over 32 elements (2^-21 of sum
    |q|); sums in the products and of groups, each off by 2^-22 of what it adds up, three deep (2^-20);
    the factor to log2 units and back, 2^-22 of the score."""
    b = q4_ref.Batch([n] * batch, [1] * batch, g=g, d=d, device=cuda)
    gen = torch.Generator().manual_seed(4)
    for s in range(batch):
        o = int(b.seq[s])
        b.k[0, :, o:o + n] = q4_ref.packed((torch.randn((2, n, d), generator=gen) + mean).bfloat16())
    b.q[:batch] = (torch.randn((batch, b.H_q, d), generator=gen) + 0.5).bfloat16()
    b.to_device()
    q = b.qd[:batch].contiguous()
    out, stats = torch.empty_like(q), torch.empty((batch, b.H_q, 4), device=cuda)
    ws = torch.empty(lg.lg_workspace_size(b.cache, b.H_q, 1, b.max_len), dtype=torch.uint8, device=cuda)
    lg.lg_decode_attend(b.cache, 0, 1, q, b.H_q, d ** -0.5, out, stats, 64, 0, b.max_len, ws)
    assert lg.lg_read_device_status(b.cache) == 0
    got, scale = stats.cpu().double()[..., 0], d ** -0.5
    for s in range(batch):
        o = int(b.seq[s])
        for h in range(b.H_q):
            c, sc, lo = q4_ref.parts(b.k[0, h // g, o:o + n])
            x = b.q[s, h].double()
            z = (c * sc + lo) @ x * scale
            err = scale * 2.0 ** -20 * ((lo.abs() @ x.abs()) + 15 * (sc @ x.abs()))
            tol = float(err.max() + 2.0 ** -22 * z.abs().max())
            assert abs(float(got[s, h]) - float(z.max())) <= tol, (s, h, float(got[s, h]), float(z.max()), tol)
