"""Queries of any size over a 4-bit cache: the row of the largest score where scores are far apart, and NaN,
not a number, from 2^121 on."""
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


def _run(cuda, d, top, m, dtype_scale=1.0):
    """(results, values of the row of the largest score, what a result may be off by), scores by 2^top"""
    b = q4_ref.Batch([150, 40], [m, 1], g=2, d=d, device=cuda)
    base = torch.randn((b.T, b.H_q, d), generator=torch.Generator().manual_seed(3))
    base /= base.abs().amax(-1, keepdim=True)        # the largest element one
    b.q = (base.double() * 2.0 ** top).float().bfloat16()
    b.to_device()
    out = torch.full_like(b.qd, 7.0)
    lg.lg_chunk_attend(b.cache, b.chunk, 0, b.qd, b.H_q, dtype_scale * d ** -0.5, 0, 0, out, b.max_len, b.ws)
    assert lg.lg_read_device_status(b.cache) == 0
    out, t = out.cpu().double(), 0
    want, tol = torch.zeros_like(out), torch.zeros_like(out)
    for o, n, mm in zip(b.seq, b.ns, b.ms):
        for h in range(b.H_q):
            K, V = b.k[0, h // 2, o:o + n], b.v[0, h // 2, o:o + n]
            score = b.q[t:t + mm, h].double() @ q4_ref.values(K).T
            for j in range(mm):
                score[j, n - mm + j + 1:] = -torch.inf
            at = score.argmax(-1)
            c, s, lo = (x[at] for x in q4_ref.parts(V))
            want[t:t + mm, h] = c * s + lo
            # one weight of one, rounded with the scale: see q4_ref
            tol[t:t + mm, h] = 2.0 ** -7 * s * (c - 8).abs() + 2.0 ** -8 * (lo + 8 * s).abs() + \
                2.0 ** -8 * (c * s + lo).abs() + 2.0 ** -17 * (s * (c - 8).abs() + lo.abs() + 8 * s)
        t += mm
    return out[:t], want[:t], tol[:t]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 4])
@pytest.mark.parametrize("top", [20, 60, 100, 113, 114, 118, 120])
def test_scores_far_apart(cuda, d, m, top):
    out, want, tol = _run(cuda, d, top, m)
    assert ((out - want).abs() <= tol).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 4])
@pytest.mark.parametrize("top,scale", [(121, 1.0), (123, 1.0), (127, 1.0), (110, 2.0 ** 10)])
def test_queries_out_of_range_show(cuda, d, m, top, scale):
    out, _, _ = _run(cuda, d, top, m, scale)
    assert torch.isnan(out).all()
