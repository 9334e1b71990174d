"""lg_chunk_attend against the 64-bit form (chunk_ref.py, where the tolerances are derived): both
element types and head sizes, every query group, lengths from none to long ones, windows and sinks
around tile and block bounds; the exact set of rows seen; rows that hold no numbers where no query
looks; its errors, streams, graphs and workspaces."""
import math

import numpy as np
import pytest
import torch

import chunk_ref
from chunk_ref import Batch, visible
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ns,ms", [
    ([1], [1]), ([17], [1]), ([300], [1]), ([1025], [1]), ([64, 128, 129, 1], [1, 1, 1, 1]),
    ([5], [5]), ([130], [130]), ([300, 0, 77], [40, 0, 77]), ([257, 600], [3, 129]),
    ([0, 0, 9, 0], [0, 0, 2, 0])])
def test_lengths(cuda, dtype, ns, ms):
    b = Batch(ns, ms, dtype, seed=len(ns) + ns[0]).to_device()
    b.check(b.attend())


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("g", [1, 2, 3, 4, 5, 6, 7, 8])
def test_query_groups(cuda, dtype, d, g):
    b = Batch([150, 200, 40], [150, 1, 33], dtype, H_kv=4 if d == 64 else 2, g=g, d=d, seed=g,
              spread=2.0).to_device()
    b.check(b.attend())
    one = Batch([150, 2, 401], [1, 1, 1], dtype, H_kv=4 if d == 64 else 2, g=g, d=d, seed=g,
                spread=2.0).to_device()
    one.check(one.attend())


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 4), (2, 1), (63, 0), (64, 4), (65, 64),
                                         (128, 130), (200, 3), (5000, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(cuda, dtype, d, window, sink):
    b = Batch([700, 130, 301, 64], [300, 130, 1, 5], dtype, d=d, seed=window % 97).to_device()
    b.check(b.attend(window, sink), window, sink)
    one = Batch([700, 130, 1, 64], [1, 1, 1, 1], dtype, d=d, seed=window % 97).to_device()
    one.check(one.attend(window, sink), window, sink)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(0, 0), (100, 0), (37, 5), (128, 64)])
@pytest.mark.parametrize("ms", [[500, 260, 129], [1, 1, 1], [9, 2, 64]])
def test_the_rows_seen_are_exactly_these(cuda, dtype, window, sink, ms):
    """all scores equal and row i's value one in element i mod d: a result is the number of rows
    seen of each residue over their total, exact before its one rounding"""
    ns = [500, 391, 130]
    b = Batch(ns, ms, dtype, seed=1)
    b.k = torch.where(b.k.isnan(), b.k, torch.zeros_like(b.k))
    for o, n in zip(b.seq, ns):
        i = torch.arange(n)
        b.v[:, :, o:o + n] = 0.0
        b.v[:, :, o + i, i % b.d] = 1.0
    b.to_device()
    out = b.attend(window, sink).double().cpu()
    assert lg.lg_read_device_status(b.cache) == 0
    t = 0
    for n, m in zip(ns, ms):
        see = visible(n, m, window, sink).double()
        count = torch.zeros(m, b.d, dtype=torch.float64)
        count.index_add_(1, torch.arange(n) % b.d, see)
        want = (count / see.sum(-1, keepdim=True))[:, None].expand(m, b.H_q, b.d)
        # one division or reciprocal and product in fp32, one rounding to the type
        step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
        assert ((out[t:t + m] - want).abs() <= want * (step + 2.0 ** -22)).all()
        t += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(0, 0), (50, 3)])
def test_what_hidden_rows_hold_is_nothing(cuda, dtype, window, sink):
    """NaN and infinities in keys and values of rows that some queries see and others do not: those
    that do not have the results of finite rows; those that see a NaN or infinite value have it.
    (Keys stay numbers where a query sees them.)"""
    ns, ms = [400, 200], [150, 1]
    b = Batch(ns, ms, dtype, seed=3)
    o = int(b.seq[0])
    b.v[:, 0, o + 300, 5] = math.inf
    b.v[:, 0, o + 340, 6] = math.nan
    b.v[:, 1, o + 399, :] = -math.inf      # only the last query sees it
    if window:                             # rows before every window, after the sinks
        b.k[:, :, o + 3:o + 200] = math.nan
        b.v[:, :, o + 3:o + 200] = math.inf
        o2 = int(b.seq[1])
        b.k[:, :, o2 + 3:o2 + 150] = math.nan
        b.v[:, :, o2 + 3:o2 + 150] = math.nan
    b.to_device()
    out = b.attend(window, sink)
    if window:  # the reference multiplies hidden rows: finite ones in their place
        b.k = torch.nan_to_num(b.k, nan=0.0)
        v = b.v.clone()
        v[:, :, o + 3:o + 200] = 0.0
        v[:, :, o2 + 3:o2 + 150] = 0.0
        b.v = v
    b.check(out, window, sink)


def _under_a_window(b, d, how):
    """the batch's scores as they are, all lower by 100, far apart, or far apart for each sequence's
    first token only (its maxima rise in later blocks, beside the others')"""
    if how == "first token":
        at = np.concatenate([[0], np.cumsum(b.ms)[:-1]])
        b.q[at] *= 12.0
    if how == "low":  # one element of every query and key makes -100 of each score
        b.q[..., 0] = 16.0
        b.k[..., 0] = torch.where(b.k[..., 0].isnan(), b.k[..., 0],
                                  torch.full_like(b.k[..., 0], -100.0 * d ** 0.5 / 16.0))
    return b.to_device()


@pytest.mark.parametrize("how", ["even", "low", "far apart", "first token"])
@pytest.mark.parametrize("d,H_kv,g,m", [(128, 2, 4, 2), (128, 2, 4, 4), (128, 1, 8, 2), (64, 2, 4, 3),
                                        (128, 2, 4, 7), (64, 2, 4, 8), (128, 1, 1, 16),
                                        (128, 2, 4, 16), (64, 4, 1, 50), (128, 1, 3, 21)])
@pytest.mark.parametrize("window,sink", [(512, 0), (1000, 4), (1024, 0), (4096, 0)])
def test_some_tokens_whose_windows_start_in_other_blocks(cuda, d, H_kv, g, m, window, sink, how):
    """a tile of few rows whose first block only some of its tokens see, in whole items and in items
    that are cut after several blocks"""
    # the first row that the tile sees stands 1 to 12 rows before a block's end
    ns = [window + m - 1 + 128 * (1 + i) + 116 + i for i in range(12)]
    b = Batch(ns, [m] * 12, "bf16", H_kv=H_kv, g=g, d=d, seed=window + m,
              spread=12.0 if how == "far apart" else 1.0)
    _under_a_window(b, d, how)
    b.check(b.attend(window, sink), window, sink)
    one = Batch(ns[5:6], [m], "bf16", H_kv=H_kv, g=g, d=d, seed=window + m,
                spread=12.0 if how == "far apart" else 1.0)
    _under_a_window(one, d, how)
    one.check(one.attend(window, sink), window, sink)


@pytest.mark.parametrize("window,sink", [(1000, 0), (1000, 4)])
def test_proposed_tokens_of_a_batch_under_a_window(cuda, window, sink):
    """16 sequences of up to 4099 rows, 32/8 heads, 7 tokens each"""
    rng = np.random.default_rng(3)
    ns = [4099] + [int(x) for x in np.exp(rng.uniform(np.log(256), np.log(4099), 15))]
    b = Batch(ns, [7] * 16, "bf16", H_kv=8, g=4, seed=17).to_device()
    b.check(b.attend(window, sink), window, sink)


@pytest.mark.parametrize("d,m", [(128, 1), (128, 5), (128, 200), (64, 1), (64, 5), (64, 200)])
def test_hidden_rows_again_and_again(cuda, d, m):
    """rows without numbers behind every window, at every place of the ring that blocks pass through:
    none of them reaches a result, in any of many calls"""
    window, ns = 300, [m + 1500 + 37 * i for i in range(24)]
    b = Batch(ns, [m] * 24, "bf16", d=d, seed=16)
    for o, n in zip(b.seq, ns):
        b.k[:, :, o:o + n - m + 1 - window] = math.nan
        b.v[:, :, o:o + n - m + 1 - window] = math.nan
    b.to_device()
    out = b.attend(window)
    for o, n in zip(b.seq, ns):  # (the reference multiplies hidden rows)
        b.k[:, :, o:o + n - m + 1 - window] = 0.0
        b.v[:, :, o:o + n - m + 1 - window] = 0.0
    b.check(out, window)
    for _ in range(20):
        assert torch.equal(out, b.attend(window))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_later_keys_that_are_not_numbers(cuda, dtype):
    """a NaN key in a later row leaves the queries before it alone"""
    b = Batch([300], [300], dtype, seed=4).to_device()
    want = b.attend()
    o = int(b.seq[0])
    b.cache.k[:, :, o + 250] = math.nan
    b.cache.v[:, :, o + 250] = math.nan
    got = b.attend()
    assert torch.equal(got[:250], want[:250])
    assert got[250:300].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(cuda, dtype):
    """scores far apart: the running maximum rises many times and most weights vanish"""
    b = Batch([600, 190], [200, 1], dtype, seed=5, spread=12.0).to_device()
    b.check(b.attend())


@pytest.mark.parametrize("dtype,m", [("bf16", 1), ("bf16", 300), ("f32", 1), ("f32", 300)])
def test_long_cache(cuda, dtype, m):
    """one long sequence shared by many CTAs"""
    b = Batch([9001], [m], dtype, H_kv=2, g=2, seed=6).to_device()
    b.check(b.attend())
    b.check(b.attend(1000, 4), 1000, 4)


@pytest.mark.parametrize("dtype,g,m", [("bf16", 1, 1), ("bf16", 8, 1), ("bf16", 5, 2),
                                       ("bf16", 8, 2), ("f32", 3, 1), ("f32", 8, 1),
                                       ("f32", 5, 3), ("f32", 8, 2)])
def test_few_rows_in_many_parts(cuda, dtype, g, m):
    """items of up to 16 rows that are cut into 9, 17 and more parts; a window that empties some"""
    for H_kv, ns in ((1, [20000]), (2, [9001]), (1, [1500, 8000]), (3, [5000, 0])):
        ms = [min(n, m) for n in ns]
        d = 64 if g == 8 and H_kv % 2 == 0 else 128  # (a cache's H_kv d is a multiple of 128)
        b = Batch(ns, ms, dtype, H_kv=H_kv, g=g, d=d, seed=14).to_device()
        out = b.attend()
        b.check(out)
        assert torch.equal(out, b.attend())
        b.check(b.attend(1200, 4), 1200, 4)
    b.v[:, :, 77, :5] = math.inf  # a value that every query sees, in one part of many
    b.to_device()
    b.check(b.attend())


def test_many_sequences(cuda):
    """more sequences than a CTA has threads, empty ones and empty chunks among them"""
    rng = np.random.default_rng(7)
    ns = [int(x) for x in rng.integers(0, 40, 700)]
    for ms in ([min(n, int(x)) for n, x in zip(ns, rng.integers(0, 5, 700))],
               [min(n, 1) for n in ns]):
        b = Batch(ns, ms, "bf16", H_kv=2, g=2, d=64, seed=8).to_device()
        b.check(b.attend())


def test_layers_and_offsets(cuda):
    """each layer of a cache by itself; a chunk that starts behind other rows"""
    b = Batch([200, 90], [30, 90], "bf16", L=3, seed=9).to_device()
    for layer in (2, 0, 1):
        b.check(b.attend(layer=layer), layer=layer)
    out0 = b.attend()
    q = torch.cat([torch.full_like(b.qd[:5], math.nan), b.qd])
    b.chunk = lg.Chunk(b.chunk.off + 5, b.T + 5, b.chunk.max_new)
    b.qd = q
    out = b.attend()
    assert torch.equal(out[5:], out0) and (out[:5] == 7.0).all()


def test_a_wider_bound_gives_the_same_answers(cuda):
    """max_new and max_len above the lengths"""
    for dtype in ("bf16", "f32"):
        b = Batch([200, 90], [1, 1], dtype, seed=10).to_device()
        b.chunk = lg.Chunk(b.chunk.off, b.T, 64)
        b.max_len = 1000
        b.ws = torch.empty(lg.lg_chunk_workspace_size(b.cache, b.chunk, b.H_q, b.max_len),
                           dtype=torch.uint8, device=cuda)
        b.check(b.attend())


@pytest.mark.parametrize("H_kv,g,d,ns,ms", [
    (2, 4, 128, [600], [600]), (4, 4, 128, [700, 300, 900], [513, 0, 64 * 9]),
    (8, 2, 64, [1100, 40, 300], [1100, 40, 129]), (6, 8, 128, [300, 290], [290, 290]),
    (8, 1, 128, [2300, 5, 2048], [2300, 5, 1792]), (8, 7, 64, [500], [300]),
    (16, 2, 64, [130] * 35 + [700], [130] * 5 + [0, 1, 90] * 10 + [640]),
    (4, 5, 128, [9] * 33 + [1000], [1] * 33 + [1000])])
def test_tiles_dealt_to_lines(cuda, H_kv, g, d, ns, ms):
    """a bound on the lengths past what the L2 holds deals a kv-head's tiles to several lines"""
    b = Batch(ns, ms, "bf16", H_kv=H_kv, g=g, d=d, seed=12).to_device()
    b.check(b.attend())
    for b.max_len in (20000, 2 ** 31 - 1):
        b.check(b.attend())


def test_tiles_dealt_to_lines_under_a_window(cuda):
    for H_kv, n, m, window, sink in ((2, 3100, 650, 1700, 4), (4, 2600, 2600, 1600, 130)):
        b = Batch([n, 50], [m, 50], "bf16", H_kv=H_kv, g=4, seed=13).to_device()
        b.check(b.attend(window, sink), window, sink)


@pytest.mark.parametrize("d,H_kv,g", [(128, 2, 4), (128, 1, 8), (64, 2, 4), (64, 4, 1)])
def test_short_last_tiles_one_after_another(cuda, d, H_kv, g):
    """pieces of one stream's tile alone, short enough that all their blocks arrive at once, followed
    by pieces of both: every piece computes with its own queries"""
    tile = 128 // g
    ms = [tile // 2, 2 * tile, tile, 1, 2 * tile - 1, 2 * tile + 3, tile + 1] * 60
    ns = [m + x for m, x in zip(ms, [0, 0, 90, 100, 0, 40, 3] * 60)]
    b = Batch(ns, ms, "bf16", H_kv=H_kv, g=g, d=d, seed=15, spread=2.0).to_device()
    out = b.attend()
    b.check(out)
    for _ in range(20):
        assert torch.equal(out, b.attend())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,m", [(3, 1), (5, 1), (6, 4), (7, 2), (4, 3), (1, 7), (5, 12), (3, 90)])
def test_rows_beside_a_tiles_queries_change_no_bit(cuda, dtype, g, m):
    """rows of a tile that are no query: what the shared memory held before the call, and the queries of
    the sequences behind"""
    ns = [1500 + 31 * i for i in range(40)]
    b = Batch(ns, [m] * 40, dtype, H_kv=2, g=g, seed=18).to_device()
    full = Batch([1500] * 40, [m] * 40, dtype, H_kv=1, g=8, seed=18).to_device()
    q, out = b.qd.clone(), b.attend()
    b.check(out)
    for value in (0.0, 300.0, -300.0, 1e30, math.inf, math.nan):
        full.qd.fill_(value)  # (its tiles' rows are queries all)
        full.attend()
        assert torch.equal(out, b.attend()), value
        b.qd[m:] = value
        assert torch.equal(out[:m], b.attend()[:m]), value
        b.qd.copy_(q)


@pytest.mark.parametrize("what", ["max_len", "max_new", "more new rows than rows", "T", "order"])
def test_lengths_out_of_bounds_are_an_error(cuda, what):
    b = Batch([200, 90], [30, 20], "bf16", seed=11).to_device()
    off = b.chunk.off.clone()
    if what == "max_len":
        b.max_len = 199
    elif what == "max_new":
        b.chunk = lg.Chunk(off, b.T, 29)
    elif what == "T":
        b.chunk = lg.Chunk(off, 49, 30)
    elif what == "order":
        off[1] = 60
        b.chunk = lg.Chunk(off, b.T, 100)
    else:
        b.cache.len[0] = 29
    out = torch.full_like(b.qd, 7.0)
    ws = torch.empty(1 << 28, dtype=torch.uint8, device=cuda)
    args = (b.cache, b.chunk, 0, b.qd, b.H_q, 0.1, 0, 0, out, b.max_len, ws)
    lg.lg_chunk_attend(*args)
    assert lg.lg_read_device_status(b.cache) == 4
    # and the call skips its work while the status is set
    b.cache.len.copy_(torch.tensor([200, 90]))
    lg.lg_chunk_attend(b.cache, lg.Chunk(lg.Chunk.of([30, 20], cuda).off, b.T, 30), 0, b.qd, b.H_q,
                       0.1, 0, 0, out, 200, ws)
    assert lg.lg_read_device_status(b.cache) == 4 and (out == 7.0).all()


def test_streams_and_repeats(cuda):
    """two calls at once on two streams, a workspace each; the same call again gives the same bits"""
    a = Batch([700, 30], [100, 30], "bf16", seed=12).to_device()
    b = Batch([300, 1200], [1, 1], "bf16", seed=13).to_device()
    wa, wb = a.attend(), b.attend()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(device=cuda), torch.cuda.Stream(device=cuda)
    for _ in range(5):
        with torch.cuda.stream(s1):
            ga = a.attend()
        with torch.cuda.stream(s2):
            gb = b.attend()
        torch.cuda.synchronize()
        assert torch.equal(ga, wa) and torch.equal(gb, wb)


@pytest.mark.parametrize("dtype,m", [("bf16", 1), ("bf16", 90), ("f32", 1), ("f32", 90)])
def test_captured_and_replayed(cuda, dtype, m):
    """a graph follows the lengths and rows that its replays find; two graphs on one workspace"""
    b = Batch([500, 300], [m, m], dtype, seed=14).to_device()
    b.max_len = 1000
    b.attend()
    out = torch.full_like(b.qd, 7.0)
    side = torch.cuda.Stream(device=cuda)
    graphs = []
    for window in (0, 64):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side, capture_error_mode="thread_local"):
            lg.lg_chunk_attend(b.cache, b.chunk, 0, b.qd, b.H_q, b.d ** -0.5, window, 2, out,
                               b.max_len, b.ws)
        graphs.append((g, window))
    for ns in ([500, 300], [499, 200], [m, 257]):
        b.cache.len.copy_(torch.tensor(ns, dtype=torch.int32))
        b.ns = ns
        for g, window in graphs:
            out.fill_(7.0)
            g.replay()
            b.check(out, window, 2)
