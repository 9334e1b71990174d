"""Single tokens of all layers of a 4-bit cache in one call, at layer counts that do not divide what the GPU
holds at once, against 64 bits; in a line and in clusters."""
import math

import numpy as np
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,batch,d,g,most", [(5, 3, 128, 4, 1500), (28, 3, 128, 4, 300), (28, 40, 64, 7, 400),
                                              (61, 9, 128, 2, 200), (5, 70, 128, 8, 300)])
def test_all_layers_at_once(cuda, L, batch, d, g, most):
    rng = np.random.default_rng(L + batch)
    ns = [int(x) for x in rng.integers(1, most, batch)]
    ns[1] = 0
    b = q4_ref.Batch(ns, [1 if n else 0 for n in ns], g=g, d=d, L=L, device=cuda).to_device()
    q = torch.randn((L, batch, b.H_q, d), generator=torch.Generator().manual_seed(1)).bfloat16()
    out = torch.full((L, batch, b.H_q, d), 7.0, dtype=torch.bfloat16, device=cuda)
    stats = torch.full((L, batch, b.H_q, 4), 7.0, device=cuda)
    ws = torch.full((lg.lg_workspace_size(b.cache, b.H_q, L, b.max_len),), 0xff, dtype=torch.uint8,
                    device=cuda)
    lg.lg_decode_attend(b.cache, 0, L, q.to(cuda), b.H_q, d ** -0.5, out, stats, 64, 0, b.max_len, ws)
    assert lg.lg_read_device_status(b.cache) == 0
    out, stats = out.cpu().double(), stats.cpu().double()
    for l in sorted({0, 1, L // 2, L - 1}):
        for s, n in enumerate(ns):
            o = int(b.seq[s])
            for h in range(b.H_q):
                if n == 0:
                    assert (out[l, s, h] == 0).all()
                    assert stats[l, s, h].tolist() == [-math.inf, 0.0, 0.0, 0.0]
                    continue
                ref, tol, st = q4_ref.attention(q[l, s, h][None], b.k[l, h // g, o:o + n],
                                                b.v[l, h // g, o:o + n], n, 1, d ** -0.5, suffix=64)
                assert ((out[l, s, h] - ref[0]).abs() <= tol[0]).all(), (l, s, h)
                assert ((stats[l, s, h] - st[0, 0]).abs() <= st[0, 1]).all(), (l, s, h)
