"""lg_pick_token and lg_count_tokens against the documented steps in fp32 and 64-bit sums.

Tokens and processed logits are exact.  pmax is 1 / s with s a sum of V exponentials of fp32
differences d: each off by |d| 2^-23 + 2^-22 of itself (the difference times log2 e, the
exponential), and |d| e^d <= 1/e, so s is off by at most V 2^-24 + 2^-20 of itself (s >= 1)."""
import math
import threading

import numpy as np
import pytest
import torch

import chunk_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


def _dev(x, cuda, dt=None):
    t = torch.as_tensor(np.ascontiguousarray(x), device=cuda)
    return t if dt is None else t.to(dt)


def _run(cuda, logits, seen=None, counts=None, penalty=None, bias=None, allowed=None, keep=True,
         in_place=False):
    """logits: device [B][V] (maybe strided); the others numpy [B][V], [B][V], [B][3], lists"""
    B, V = logits.shape
    args = [None, None, None]
    if seen is not None:
        pen = np.zeros((B, 4), dtype=np.float32)
        pen[:, :3] = penalty
        args = [_dev(np.stack([chunk_ref.pack(s) for s in seen]), cuda),
                _dev(counts.astype(np.int32), cuda), _dev(pen, cuda)]
    bs = None
    if bias is not None:
        off = np.concatenate([[0], np.cumsum([len(x) for x in bias])]).astype(np.int32)
        flat = [e for x in bias for e in x] + [(0, 0.0)]
        bs = (_dev(off, cuda), _dev(np.array([e[0] for e in flat], dtype=np.int32), cuda),
              _dev(np.array([e[1] for e in flat], dtype=np.float32), cuda))
    al = None if allowed is None else _dev(np.stack([chunk_ref.pack(a) for a in allowed]), cuda)
    host = logits.float().cpu().numpy()
    tok = torch.full((B,), -9, dtype=torch.int32, device=cuda)
    pm = torch.full((B,), -9.0, device=cuda)
    out = logits if in_place else torch.empty_strided(logits.shape, logits.stride(),
                                                      dtype=logits.dtype, device=cuda) if keep else None
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    lg.lg_pick_token(logits, *args, bs, al, tok, pm, status, out)
    torch.cuda.synchronize()
    assert status.item() == 0
    for b in range(B):
        t, p, x = chunk_ref.pick(host[b], None if seen is None else seen[b],
                                 None if counts is None else counts[b],
                                 None if penalty is None else penalty[b],
                                 None if bias is None else bias[b],
                                 None if allowed is None else allowed[b])
        assert tok[b].item() == t, (b, tok[b].item(), t, x[tok[b].item()], x[t])
        assert abs(pm[b].item() - p) <= p * (V * 2.0 ** -24 + 2.0 ** -20), (b, pm[b].item(), p)
        if out is not None:
            want = torch.as_tensor(x).to(logits.dtype).float()
            assert torch.equal(out[b].float().cpu(), want), b
    return tok, pm


def _history(rng, B, V, n):
    seen = np.zeros((B, V), dtype=bool)
    counts = np.zeros((B, V), dtype=np.int64)
    for b in range(B):
        ids = rng.integers(0, V, n)
        seen[b, ids] = True
        np.add.at(counts[b], ids[n // 2:], 1)
    pen = rng.random((B, 3)).astype(np.float32) + np.array([0.7, -0.3, -0.2], dtype=np.float32)
    return seen, counts, pen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", [(1, 1), (2, 7), (1, 31), (3, 33), (5, 1000), (2, 4099),
                                 (1, 50257), (3, 131072), (1, 151936), (40, 8191), (200, 513)])
def test_sizes(cuda, dtype, B, V):
    rng = np.random.default_rng(B * V)
    x = _dev(rng.standard_normal((B, V)).astype(np.float32) * 3, cuda, chunk_ref.tdtype(dtype))
    _run(cuda, x)
    seen, counts, pen = _history(rng, B, V, min(V, 300))
    bias = [[(int(t), float(v)) for t, v in zip(rng.integers(0, V, 9), rng.standard_normal(9) * 4)]
            for _ in range(B)]
    allowed = rng.random((B, V)) < 0.6
    _run(cuda, x, seen, counts, pen, bias, allowed)
    _run(cuda, x, seen, counts, pen, keep=False)
    _run(cuda, x, allowed=allowed, bias=bias)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", [(4, 90001), (8, 90001), (30, 40961), (60, 33001), (100, 24577),
                                 (150, 16385), (200, 24577), (310, 8193), (306, 90113)])
def test_rows_split_over_ctas(cuda, dtype, B, V):
    """every number of CTAs a row, and more rows than run at once"""
    rng = np.random.default_rng(B)
    x = _dev(rng.standard_normal((B, V), dtype=np.float32) * 3, cuda, chunk_ref.tdtype(dtype))
    seen, counts, pen = _history(rng, B, V, 300)
    _run(cuda, x, seen, counts, pen, None, rng.random((B, V), dtype=np.float32) < 0.6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [3, 96])
def test_many_seen_tokens(cuda, dtype, B):
    """histories that fill stretches of the vocabulary, more of them than a CTA lists"""
    V = 60013
    rng = np.random.default_rng(B)
    x = _dev(rng.standard_normal((B, V)).astype(np.float32) * 3, cuda, chunk_ref.tdtype(dtype))
    seen, counts, pen = _history(rng, B, V, 4000)
    seen[:, 100:9000] = True
    counts[:, 200:5000] += rng.integers(0, 3, (B, 4800))
    bias = [[(int(t), 1.5) for t in rng.integers(0, V, 5)] for _ in range(B)]
    _run(cuda, x, seen, counts, pen, bias)
    _run(cuda, x, seen, counts, pen, bias, rng.random((B, V)) < 0.5)
    _run(cuda, x, seen, counts, pen, bias, in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [3, 200])
def test_seen_and_biased_beside_many_seen_tokens(cuda, dtype, B):
    """more seen tokens than a CTA lists, and behind them seen tokens that stand alone in their word of
    bits and are biased: each counts once, with its bias, however far up it was or is moved"""
    V = 60013
    rng = np.random.default_rng(B)
    host = rng.standard_normal((B, V)).astype(np.float32) * 3
    alone = np.arange(2600, 3600, 100)
    host[:, alone[:5]] = 60.0              # on top but for their bias
    x = _dev(host, cuda, chunk_ref.tdtype(dtype))
    seen, counts = np.zeros((B, V), dtype=bool), np.zeros((B, V), dtype=np.int64)
    seen[:, :2500] = True
    seen[:, alone] = True
    counts[:, 1000:2000] = rng.integers(0, 3, (B, 1000))
    counts[:, alone[::2]] = 2
    pen = rng.random((B, 3)).astype(np.float32) + np.array([1.0, 0.0, 0.0], dtype=np.float32)
    low = [[(int(t), -100.0) for t in alone] for _ in range(B)]
    high = [[(int(t), 40.0) for t in alone[5:]] + [(int(t), -100.0) for t in alone[:5]]
            for _ in range(B)]
    for bias in (low, high):
        _run(cuda, x, seen, counts, pen, bias)
        _run(cuda, x, seen, counts, pen, bias, keep=False)
        _run(cuda, x.clone(), seen, counts, pen, bias, in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_in_place(cuda, dtype):
    rng = np.random.default_rng(1)
    for V, pad in ((1001, 6), (777, 0), (640, 3)):
        for shift in (0, 1, 3):  # rows at every alignment
            buf = torch.randn((7, V + pad + shift), device=cuda).to(chunk_ref.tdtype(dtype))
            x = buf[:, shift:shift + V]
            keep = buf.clone()
            seen, counts, pen = _history(rng, 7, V, 100)
            allowed = rng.random((7, V)) < 0.5
            _run(cuda, x, seen, counts, pen, None, allowed)
            assert torch.equal(buf, keep)
            _run(cuda, x, seen, counts, pen, None, allowed, in_place=True)
            assert torch.equal(buf[:, :shift], keep[:, :shift])
            assert torch.equal(buf[:, shift + V:], keep[:, shift + V:])


def test_ties_go_to_the_lowest_token(cuda):
    for V in (100, 5000, 140001):
        x = torch.zeros((4, V), device=cuda)
        for b, ids in enumerate(([V - 1, 0], [V // 2, V // 2 + 1, V - 1], [17], list(range(V)))):
            x[b, ids] = 2.5
        _run(cuda, x)
        _run(cuda, x.bfloat16())


def test_rows_with_nothing_left_and_infinities(cuda):
    V = 9000
    x = torch.randn((6, V), device=cuda)
    allowed = np.ones((6, V), dtype=bool)
    allowed[0] = False
    allowed[1] = False
    allowed[1, V - 1] = True
    x[1, V - 1] = -50.0
    x[2] = -math.inf
    x[3, 5] = math.nan
    x[3, 100:] = math.nan
    x[4, [70, 8000]] = math.inf
    x[5] = float(torch.finfo(torch.float32).min)
    tok, pm = _run(cuda, x, allowed=allowed)
    assert tok[0].item() == -1 and pm[0].item() == 0.0 and tok[1].item() == V - 1
    assert pm[1].item() == 1.0 and tok[2].item() == -1 and pm[4].item() == 0.5
    _run(cuda, x.bfloat16(), allowed=allowed)


def test_large_vocabulary_and_batch(cuda):
    """a row's bits take several CTAs' shared memory although the batch alone fills the GPU"""
    B, V = 400, 350003
    x = torch.zeros((B, V), dtype=torch.bfloat16, device=cuda)
    at = torch.arange(B, device=cuda) * 875 % V
    x[torch.arange(B, device=cuda), at] = 3.0
    tok = torch.zeros(B, dtype=torch.int32, device=cuda)
    pm = torch.zeros(B, device=cuda)
    lg.lg_pick_token(x, None, None, None, None, None, tok, pm)
    assert torch.equal(tok.long(), at)
    want = 1.0 / (1.0 + (V - 1) * math.exp(-3.0))
    assert ((pm - want).abs() <= want * (V * 2.0 ** -24 + 2.0 ** -20)).all()
    x = torch.zeros((2, 1 << 20), device=cuda)     # the largest vocabulary
    x[0, -1] = x[1, 777777] = 1.0
    lg.lg_pick_token(x, None, None, None, None, None, tok[:2], pm[:2])
    assert tok[:2].tolist() == [(1 << 20) - 1, 777777]


@pytest.mark.parametrize("B,V", [(180, 626688), (180, 626689), (170, 900001), (140, 500001)])
def test_divisions_of_large_vocabularies(cuda, B, V):
    """rows on both sides of what leaves room for two CTAs' bits an SM"""
    x = torch.zeros((B, V), dtype=torch.bfloat16, device=cuda)
    at = torch.arange(B, device=cuda) * 3001 % V
    x[torch.arange(B, device=cuda), at] = 3.0
    tok = torch.zeros(B, dtype=torch.int32, device=cuda)
    pm = torch.zeros(B, device=cuda)
    lg.lg_pick_token(x, None, None, None, None, None, tok, pm)
    assert torch.equal(tok.long(), at)
    want = 1.0 / (1.0 + (V - 1) * math.exp(-3.0))
    assert ((pm - want).abs() <= want * (V * 2.0 ** -24 + 2.0 ** -20)).all()


def test_calls_of_several_threads(cuda):
    """rows whose bits take different amounts of shared memory, from host threads at once"""
    def calls(V, errors):
        try:
            s = torch.cuda.Stream(device=cuda)
            with torch.cuda.stream(s):
                x = torch.zeros((310, V), dtype=torch.bfloat16, device=cuda)
                x[:, V - 7] = 2.0
                tok = torch.zeros(310, dtype=torch.int32, device=cuda)
                pm = torch.zeros(310, device=cuda)
                status = torch.ones(1, dtype=torch.int32, device=cuda)  # (the work is skipped)
                for _ in range(20000):
                    lg.lg_pick_token(x, None, None, None, None, None, tok, pm, status)
                status.zero_()
                lg.lg_pick_token(x, None, None, None, None, None, tok, pm, status)
                assert (tok == V - 7).all()
        except Exception as e:
            errors.append(e)

    errors = []
    threads = [threading.Thread(target=calls, args=(V, errors)) for V in (150000, 90000, 250000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors


def test_bias_lists(cuda):
    """empty lists, one token twice, tokens outside the vocabulary, long lists"""
    V = 3001
    x = torch.randn((4, V), device=cuda)
    rng = np.random.default_rng(3)
    bias = [[], [(5, 2.0), (5, 7.25), (5, -1.5)], [(-1, 99.0), (V, 99.0), (V - 1, 9.0), (2 ** 30, 99.0)],
            [(int(t), float(v)) for t, v in zip(rng.integers(0, V, 2000), rng.standard_normal(2000))]]
    _run(cuda, x, bias=bias)


@pytest.mark.parametrize("B,V", [(1, 151936), (16, 60013), (200, 33001)])
def test_the_same_call_gives_the_same_bits(cuda, B, V):
    """listed tokens, more of them than are listed, and biased ones, some repeatedly: the sums are taken
    in one order"""
    rng = np.random.default_rng(V)
    x = torch.randn((B, V), device=cuda)
    for n, lists in ((1500, 0), (1500, 200), (30000, 200)):
        seen, counts, pen = _history(rng, B, V, n)
        args = [_dev(np.stack([chunk_ref.pack(s) for s in seen]), cuda),
                _dev(counts.astype(np.int32), cuda),
                _dev(np.concatenate([pen, np.zeros((B, 1), dtype=np.float32)], 1), cuda)]
        bias = None
        if lists:
            ids = rng.integers(0, V, (B, lists))
            ids[:, lists // 2:] = ids[:, :lists // 2]      # each of them twice
            bias = (_dev(np.arange(0, B * lists + 1, lists, dtype=np.int32), cuda),
                    _dev(ids.reshape(-1).astype(np.int32), cuda), torch.randn(B * lists, device=cuda))
        tok = torch.zeros((30, B), dtype=torch.int32, device=cuda)
        pm = torch.zeros((30, B), device=cuda)
        for i in range(30):
            lg.lg_pick_token(x, *args, bias, None, tok[i], pm[i])
        assert (tok == tok[0]).all() and (pm == pm[0]).all(), (n, lists)


def test_count_tokens(cuda):
    V, B = 1003, 3
    nw = (V + 31) // 32
    seen = torch.zeros((B, nw), dtype=torch.int32, device=cuda)
    counts = torch.zeros((B, V), dtype=torch.int32, device=cuda)
    want_s, want_c = np.zeros((B, V), dtype=bool), np.zeros((B, V), dtype=np.int64)
    rng = np.random.default_rng(2)
    rows = [rng.integers(0, V, 400), rng.integers(-5, V + 5, 0), np.full(70000, 17)]
    rows[0][:50] = 31
    for generated in (0, 1):
        off = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int32)
        ids = np.concatenate(rows + [[-1, V, 2 ** 31 - 1]]).astype(np.int32)
        off[-1] += 2  # the last row ends with a token of -1 and one past the vocabulary
        lg.lg_count_tokens(_dev(ids, cuda), _dev(off, cuda), V, generated, seen, counts)
        for b, r in enumerate(rows):
            want_s[b, r] = True
            if generated:
                np.add.at(want_c[b], r, 1)
    step = np.array([5, -1, 17], dtype=np.int32)
    lg.lg_count_tokens(_dev(step, cuda), None, V, 1, seen, counts)
    want_s[0, 5] = True
    want_c[0, 5] += 1
    want_c[2, 17] += 1
    assert np.array_equal(counts.cpu().numpy(), want_c)
    assert np.array_equal(seen.cpu().numpy(), np.stack([chunk_ref.pack(s) for s in want_s]))


def test_count_as_many_tokens_as_fit(cuda):
    """2^31 - 10 tokens, most of them none of the vocabulary"""
    T, V = 2 ** 31 - 10, 40
    tokens = torch.full((T,), -1, dtype=torch.int32, device=cuda)
    tokens[-3:] = torch.tensor([7, 39, 7], dtype=torch.int32)
    off = torch.tensor([0, T - 1, T], dtype=torch.int32, device=cuda)
    seen = torch.zeros((2, 2), dtype=torch.int32, device=cuda)
    counts = torch.zeros((2, V), dtype=torch.int32, device=cuda)
    lg.lg_count_tokens(tokens, off, V, 1, seen, counts)
    want = torch.zeros((2, V), dtype=torch.int32)
    want[0, [7, 39]] = 1
    want[1, 7] = 1
    assert torch.equal(counts.cpu(), want)
    assert seen.tolist() == [[1 << 7, 1 << 7], [1 << 7, 0]]


def test_status_and_streams_and_graphs(cuda):
    V = 20000
    x = torch.randn((2, V), device=cuda)
    tok = torch.full((2,), -9, dtype=torch.int32, device=cuda)
    pm = torch.full((2,), -9.0, device=cuda)
    status = torch.full((1,), 4, dtype=torch.int32, device=cuda)
    seen = torch.zeros((2, V // 32), dtype=torch.int32, device=cuda)
    counts = torch.zeros((2, V), dtype=torch.int32, device=cuda)
    lg.lg_pick_token(x, None, None, None, None, None, tok, pm, status)
    lg.lg_count_tokens(tok, None, V, 1, seen, counts, status)
    assert (tok == -9).all() and (pm == -9.0).all()
    status.zero_()
    side = torch.cuda.Stream(device=cuda)
    torch.cuda.synchronize()
    pen = torch.tensor([[1.3, 0.1, 0.2, 0.0]] * 2, device=cuda)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side, capture_error_mode="thread_local"):
        lg.lg_pick_token(x, seen, counts, pen, None, None, tok, pm, status)
        lg.lg_count_tokens(tok, None, V, 1, seen, counts, status)
    s, c = np.zeros((2, V), dtype=bool), np.zeros((2, V), dtype=np.int64)
    host = x.cpu().numpy()
    for _ in range(8):  # the picked token is penalised, so another comes to the top in time
        g.replay()
        torch.cuda.synchronize()
        for b in range(2):
            t, _, _ = chunk_ref.pick(host[b], s[b], c[b], [1.3, 0.1, 0.2], None, None)
            assert tok[b].item() == t
            s[b, t] = True
            c[b, t] += 1
    assert len(np.nonzero(c[0])[0]) > 1
