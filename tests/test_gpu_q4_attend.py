"""Attention over a 4-bit cache against 64 bits: single tokens with the guard's statistics, a few drafted
tokens, chunks, windows, rows that hold no numbers."""
import math

import numpy as np
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


def _check(b, window=0, sink=0):
    wide = max(b.ms) * b.g > 64
    out = b.attend(window, sink).cpu().double()
    assert lg.lg_read_device_status(b.cache) == 0
    ref, tol = b.reference(window, sink, wide)
    bad = ~((out - ref).abs() <= tol)
    assert not bad.any(), (bad.nonzero()[:5].tolist(), (out - ref)[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [1, 3, 4, 7, 8])
@pytest.mark.parametrize("ns,ms", [
    ([1], [1]), ([15, 16, 17], [1, 1, 1]), ([64, 65, 129], [1, 1, 0]), ([1000], [1]),
    ([5, 40, 333], [5, 2, 4]), ([700, 3, 64], [7, 3, 1])])
def test_few_rows(cuda, d, g, ns, ms):
    _check(q4_ref.Batch(ns, ms, g=g, d=d, device=cuda).to_device())


@pytest.mark.parametrize("d,g", [(64, 7), (128, 4)])
@pytest.mark.parametrize("window,sink", [(1, 0), (3, 1), (64, 0), (100, 4), (130, 70), (5000, 2)])
def test_windows(cuda, d, g, window, sink):
    _check(q4_ref.Batch([300, 1, 900, 77], [4, 1, 2, 0], g=g, d=d, device=cuda).to_device(), window, sink)


@pytest.mark.parametrize("d,g,most", [(64, 1, 1), (128, 4, 1), (64, 7, 4), (128, 2, 8), (128, 5, 5),
                                      (128, 4, 13)])
@pytest.mark.parametrize("window,sink", [(0, 0), (90, 5)])
def test_many_sequences_in_one_line(cuda, d, g, most, window, sink):
    """more items than clusters: CTAs whose share begins and ends inside items, empty sequences among
    them"""
    rng = np.random.default_rng(most)
    ns = [int(x) for x in rng.integers(0, 700, 45)]
    ns[3], ns[7], ns[44] = 1, 0, 1500
    ms = [int(min(n, rng.integers(0, most + 1))) if most > 1 else int(n > 0) for n in ns]
    ms[44] = most
    _check(q4_ref.Batch(ns, ms, g=g, d=d, device=cuda).to_device(), window, sink)


@pytest.mark.parametrize("d,g,most,count", [(64, 1, 1, 20), (64, 2, 3, 110), (128, 1, 1, 200),
                                            (128, 3, 1, 300), (64, 8, 2, 30), (64, 3, 5, 70)])
def test_items_of_every_division(cuda, d, g, most, count):
    """as many items as give clusters of eight CTAs, of two, single ones, and a line"""
    rng = np.random.default_rng(count)
    ns = [int(x) for x in rng.integers(0, 300, count)]
    ms = [int(min(n, rng.integers(0, most + 1))) if most > 1 else int(n > 0) for n in ns]
    ns[0], ms[0] = 301, most
    _check(q4_ref.Batch(ns, ms, g=g, d=d, device=cuda).to_device())


@pytest.mark.parametrize("d,g", [(64, 8), (128, 4), (128, 1)])
@pytest.mark.parametrize("window,sink", [(0, 0), (50, 3)])
def test_chunks(cuda, d, g, window, sink):
    """rows that take several tiles, and chunks that go through values of 16 bits"""
    for ms in ([9, 16, 2], [64, 64, 0], [150, 1, 70], [257, 200, 3]):
        b = q4_ref.Batch([400, 200, 90], ms, g=g, d=d, device=cuda).to_device()
        _check(b, window, sink)


def test_long_rows_over_many_ctas(cuda):
    for m, g in ((1, 4), (6, 4)):
        _check(q4_ref.Batch([9001, 4097], [m, m], H_kv=1, g=g, device=cuda, spread=3.0).to_device())


def test_two_layers_and_large_scores(cuda):
    _check(q4_ref.Batch([200, 90], [2, 1], L=3, layer=1, device=cuda, spread=20.0).to_device())


@pytest.mark.parametrize("d", [64, 128])
def test_a_row_without_numbers_reaches_those_that_see_it(cuda, d):
    """what a hidden row holds never reaches a result; a group of NaN among the values reaches its own
    elements, in the queries that see the row; one among the keys all of them"""
    b = q4_ref.Batch([100, 50], [4, 1], d=d, device=cuda)
    o = int(b.seq[0])
    b.v[0, 0, o + 98, d // 2:d // 2 + 4] = torch.tensor([0xff, 0x7f, 0, 0], dtype=torch.uint8)
    b.k[0, 1, o + 97, d // 2 + 4:d // 2 + 8] = torch.tensor([0xff, 0x7f, 0, 0], dtype=torch.uint8)
    out = b.to_device().attend().cpu().double()
    ref, tol = b.reference()
    nan = torch.isnan(ref)
    assert nan.any()
    # queries 2, 3 of sequence 0 see the values of row 98, 1 .. 3 the keys of row 97
    want = torch.zeros_like(nan)
    want[2:4, :4, :d // 4] = True
    want[1:4, 4:] = True
    assert torch.equal(torch.isnan(out), want)
    fine = ~want
    clean = q4_ref.Batch([100, 50], [4, 1], d=d, device=cuda)
    ref, tol = clean.reference()
    assert ((out - ref).abs() <= tol)[fine].all()


@pytest.mark.parametrize("d,g,batch", [(128, 2, 1), (128, 4, 5), (64, 7, 3), (64, 8, 70), (128, 8, 9), (64, 1, 250)])
def test_single_tokens_with_statistics(cuda, d, g, batch):
    gen = np.random.default_rng(batch)
    ns = [int(x) for x in gen.integers(1, 1500 if batch < 20 else 200, batch)]
    if batch > 3:
        ns[1], ns[3] = 0, 1
    L = 2
    b = q4_ref.Batch([max(n, 0) for n in ns], [1 if n else 0 for n in ns], g=g, d=d, L=L, device=cuda)
    b.to_device()
    q = torch.randn((L, batch, b.H_q, d), generator=torch.Generator().manual_seed(1)).bfloat16()
    out = torch.full((L, batch, b.H_q, d), 7.0, dtype=torch.bfloat16, device=cuda)
    stats = torch.full((L, batch, b.H_q, 4), 7.0, device=cuda)
    size = lg.lg_workspace_size(b.cache, b.H_q, L, b.max_len)
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device=cuda)
    lg.lg_decode_attend(b.cache, 0, L, q.to(cuda), b.H_q, d ** -0.5, out, stats, 64, 0, b.max_len, ws)
    assert lg.lg_read_device_status(b.cache) == 0
    out, stats = out.cpu().double(), stats.cpu().double()
    for l in range(L):
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
                assert ((stats[l, s, h] - st[0, 0]).abs() <= st[0, 1]).all(), \
                    (l, s, h, n, stats[l, s, h], st)
    # one layer at a time: the same within the division's order of sums, and noalloc
    one = torch.empty((1, batch, b.H_q, d), dtype=torch.bfloat16, device=cuda)
    ost = torch.empty((1, batch, b.H_q, 4), device=cuda)
    lg.lg_decode_attend_noalloc(b.cache, 1, 1, q[1:].to(cuda), b.H_q, d ** -0.5, one, ost, 64, 0,
                                b.max_len)
    assert torch.allclose(one[0].cpu().double(), out[1], rtol=2.0 ** -6, atol=2.0 ** -8)
    fine = torch.isfinite(stats[1])
    assert torch.allclose(ost[0].cpu().double()[fine], stats[1][fine], rtol=1e-5, atol=1e-5)


def test_repeated_and_captured_calls_give_the_same_bits(cuda):
    b = q4_ref.Batch([800, 3, 1500], [3, 1, 2], device=cuda).to_device()
    first = b.attend()
    assert torch.equal(b.attend(), first)
    out = torch.full_like(b.qd, 7.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lg.lg_chunk_attend(b.cache, b.chunk, 0, b.qd, b.H_q, b.d ** -0.5, 0, 0, out, b.max_len, b.ws)
    for _ in range(3):
        out.fill_(7.0)
        g.replay()
        assert torch.equal(out, first)


def test_lengths_out_of_bounds_are_reported(cuda):
    b = q4_ref.Batch([100, 50], [2, 1], device=cuda).to_device()
    b.max_len = 99
    b.attend()
    assert lg.lg_read_device_status(b.cache) == 4
    b = q4_ref.Batch([100, 50], [2, 1], device=cuda).to_device()
    b.chunk = lg.Chunk(b.chunk.off, b.T, 1)
    b.attend()
    assert lg.lg_read_device_status(b.cache) == 4
