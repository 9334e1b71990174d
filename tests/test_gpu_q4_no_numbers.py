"""A group of values of a 4-bit row that holds no numbers, in rows whose weight is below the least fp32
number: 0 times NaN is NaN in every query that sees the row and in none that does not, wherever the row
lies (in a block of which every query sees all, or in one that hides rows)."""
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


def _batch(cuda, ns, ms, d, g, at):
    """queries all alike; in sequence 0 row at is opposite to them and its values' group 0 is NaN"""
    b = q4_ref.Batch(ns, ms, g=g, d=d, device=cuda)
    gen = torch.Generator().manual_seed(5)
    base = torch.randn(d, generator=gen)
    b.q[:sum(ms)] = (8 * base).bfloat16()
    o = int(b.seq[0])
    b.k[0, :, o + at] = q4_ref.packed((-8 * base).bfloat16())
    b.v[0, :, o + at, d // 2:d // 2 + 4] = torch.tensor([0xff, 0x7f, 0, 0], dtype=torch.uint8)
    return b.to_device()


@pytest.mark.parametrize("d,g", [(64, 3), (128, 1), (128, 4)])
@pytest.mark.parametrize("n,m,at", [(20, 1, 3), (200, 1, 3), (200, 1, 199), (200, 1, 170), (60, 4, 3), (60, 4, 58),
                                    (300, 7, 40), (300, 7, 295), (400, 70, 10), (400, 70, 350)])
@pytest.mark.parametrize("window,sink", [(0, 0), (50, 2)])
def test_a_weight_of_nothing(cuda, d, g, n, m, at, window, sink):
    b = _batch(cuda, [n, 33], [m, 1], d, g, at)
    out = b.attend(window, sink).cpu().double()
    assert lg.lg_read_device_status(b.cache) == 0
    want = torch.zeros_like(out, dtype=torch.bool)
    for j in range(m):
        r = n - m + j
        if at <= r and (not window or at > r - window or at < sink):
            want[j, :, :d // 4] = True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,at", [(20, 3), (200, 3), (200, 199), (5000, 4990), (5000, 100)])
def test_single_tokens(cuda, d, n, at):
    b = _batch(cuda, [n, 33], [1, 1], d, 4, at)
    q = b.qd[:2].contiguous()
    out = torch.empty_like(q)
    stats = torch.empty((2, b.H_q, 4), device=cuda)
    ws = torch.empty(lg.lg_workspace_size(b.cache, b.H_q, 1, b.max_len), dtype=torch.uint8, device=cuda)
    lg.lg_decode_attend(b.cache, 0, 1, q, b.H_q, d ** -0.5, out, stats, 64, 0, b.max_len, ws)
    assert lg.lg_read_device_status(b.cache) == 0
    want = torch.zeros_like(out, dtype=torch.bool)
    want[0, :, :d // 4] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.isfinite(stats).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,n", [(2, 700), (2, 6000), (120, 700)])  # clusters, and lines
def test_a_part_of_nothing(cuda, d, batch, n):
    """all rows of a stretch that warps, or CTAs, take by themselves weigh nothing"""
    b = q4_ref.Batch([n] * batch, [1] * batch, g=2, d=d, device=cuda)
    base = torch.randn(d, generator=torch.Generator().manual_seed(5))
    b.q[:batch] = (8 * base).bfloat16()
    o, at = int(b.seq[1]), 200
    b.k[0, :, o + 64:o + 500] = q4_ref.packed((-8 * base).bfloat16())
    b.v[0, :, o + at, d // 2 + 8:d // 2 + 12] = torch.tensor([0xff, 0x7f, 0, 0], dtype=torch.uint8)
    out = b.to_device().attend()
    assert lg.lg_read_device_status(b.cache) == 0
    want = torch.zeros_like(out, dtype=torch.bool)
    want[1, :, d // 2:d // 2 + d // 4] = True
    assert torch.equal(torch.isnan(out), want)
