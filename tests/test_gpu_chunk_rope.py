"""lg_begin_chunk and lg_rope_append against the formulas in 64 bits.

Tolerance: an angle is exact modulo a turn up to its conversion to fp32, at most an eighth of a turn
(off by 2^-25 half turns of 2^-2: 2 pi 2^-28 radians at most), sine and cosine by 2^-22 of one
together with mscale; a rotated element is two products and a sum, off by three roundings 2^-24, so
|d| <= 2^-21 mscale (|x| + |y|) before the one rounding to the type; and the frequencies of the
formula, 2^-52 of an angle of at most 2^31."""
import numpy as np
import pytest
import torch

import chunk_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu

FAR = 2 ** 31 - 70000


def _case(dtype, d, H_q, H_kv, held, ms, cuda, seed=0, policy="loopguard", packed=True, L=2,
          pos0=None):
    rng = torch.Generator(device=cuda)
    rng.manual_seed(seed)
    dt = chunk_ref.tdtype(dtype)
    cap = np.array([n + m + 1 for n, m in zip(held, ms)], dtype=np.int32)
    off = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
    S = int(cap.sum())
    k = torch.full((L, H_kv, S, d), 3.0, dtype=dt, device=cuda)
    v = torch.full((L, H_kv, S, d), 3.0, dtype=dt, device=cuda)
    cache = lg.Cache(L, H_kv, d, dtype, off, cap, np.array(held, dtype=np.int32), cuda, policy, k, v)
    T = sum(ms) + 2  # two rows behind the last sequence
    ch = lg.Chunk.of(ms, cuda)
    ch = lg.Chunk(ch.off, T, max(ms))
    if packed:
        x = torch.randn((T, H_q + 2 * H_kv, d), generator=rng, device=cuda).to(dt)
        q, kn, vn = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    else:
        q, kn, vn = (torch.randn((T, h, d), generator=rng, device=cuda).to(dt)
                     for h in (H_q, H_kv, H_kv))
    pos = np.zeros(T, dtype=np.int32)
    t = 0
    for i, m in enumerate(ms):
        pos[t:t + m] = (held[i] if pos0 is None else pos0) + np.arange(m)
        t += m
    return cache, ch, q, kn, vn, torch.as_tensor(pos, device=cuda), off


def _np(x):
    return x.double().cpu().numpy()


def _close(got, x, pos, rp, dtype, what):
    """got [T][H][d] against x rotated"""
    want = chunk_ref.rotate(x, pos, rp)
    # |x| + |y| of the pair that an element belongs to
    mag = np.abs(x).copy()
    if rp.layout == lg.LG_ROPE_HALF:
        s = mag[..., :rp.rot // 2] + mag[..., rp.rot // 2:rp.rot]
        mag[..., :rp.rot // 2], mag[..., rp.rot // 2:rp.rot] = s, s
    else:
        s = mag[..., 0:rp.rot:2] + mag[..., 1:rp.rot:2]
        mag[..., 0:rp.rot:2], mag[..., 1:rp.rot:2] = s, s
    angle = np.abs(np.asarray(pos, dtype=np.float64)).max() * 2.0 ** -52 * 8
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = half * np.abs(want) + (2.0 ** -21 + angle) * rp.mscale * mag * (1 + half)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])
    assert np.array_equal(got[..., rp.rot:], x[..., rp.rot:]), what


def _check(case, rp, dtype, layer=1, q_out=None):
    cache, ch, q, kn, vn, pos, off = case
    H_kv, d = cache.H_kv, cache.d
    k0, v0 = cache.k.clone(), cache.v.clone()
    lens0 = cache.lengths()
    p = lg.lg_default_params(guard_layer=layer)
    if cache.sketch is not None:
        cache.sketch.fill_(-7)
    if cache.pos is not None:
        cache.pos.fill_(-7)
        cache.h2o.fill_(-7.0)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=q.device) if q_out is None else q_out
    qn, kx, vx = _np(q), _np(kn), _np(vn)
    lg.lg_begin_chunk(cache, ch)
    lg.lg_rope_append(cache, ch, layer, q, kn, vn, pos, rp, out, p)
    assert lg.lg_read_device_status(cache) == 0
    offs = ch.off.cpu().numpy()
    n = int(offs[-1])
    ps = pos.cpu().numpy()
    got = _np(out)
    _close(got[:n], qn[:n], ps[:n], rp, dtype, "q")
    if q_out is None:
        assert (got[n:] == 7.0).all(), "rows behind the last sequence"
    K, V = cache.k[layer].transpose(0, 1), cache.v[layer].transpose(0, 1)   # [S][H][d]
    touched = np.zeros(cache.S_total, dtype=bool)
    for b in range(cache.batch):
        m = offs[b + 1] - offs[b]
        assert cache.lengths()[b] == lens0[b] + m
        rows = off[b] + lens0[b] + np.arange(m)
        touched[rows] = True
        tok = np.arange(offs[b], offs[b + 1])
        if m == 0:
            continue
        _close(_np(K)[rows], kx[tok], ps[tok], rp, dtype, "k")
        assert np.array_equal(_np(V)[rows], vx[tok]), "v"
        if cache.sketch is not None:
            bits = torch.signbit(vn[torch.as_tensor(tok, device=vn.device)]).reshape(m, -1).cpu().numpy()
            want = np.stack([chunk_ref.pack(r) for r in bits])
            assert np.array_equal(cache.sketch.cpu().numpy()[rows], want), "sketch"
        if cache.pos is not None:
            assert (cache.pos[layer].cpu().numpy()[:, rows] == ps[tok]).all()
            assert (cache.h2o[layer].cpu().numpy()[:, rows] == 0).all()
    other = torch.as_tensor(~touched, device=K.device)
    for now, was in ((cache.k, k0), (cache.v, v0)):
        assert torch.equal(now[layer][:, other], was[layer][:, other])
        assert torch.equal(now[1 - layer], was[1 - layer])
    if cache.sketch is not None:
        assert (cache.sketch[other] == -7).all()
    if cache.pos is not None:
        assert (cache.pos[1 - layer] == -7).all() and (cache.pos[layer][:, other] == -7).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("part", [1, 2, 4])
def test_layouts_and_parts(cuda, dtype, d, layout, part):
    rp = lg.lg_default_rope_params(d, layout=layout, rot=d // part)
    case = _case(dtype, d, 8, 2, [5, 0, 100], [3, 40, 1], cuda, seed=part, packed=part == 2)
    _check(case, rp, dtype)


@pytest.mark.parametrize("rot", [16, 48, 80, 112])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_parts(cuda, dtype, rot):
    for layout in (0, 1):
        rp = lg.lg_default_rope_params(128, layout=layout, rot=rot)
        _check(_case(dtype, 128, 3, 1, [5], [9], cuda, seed=rot), rp, dtype)


@pytest.mark.parametrize("over", [
    dict(scaling=1, factor=8.0), dict(scaling=2, factor=4.0), dict(scaling=3, factor=8.0),
    dict(scaling=3, factor=3.0, low=0.5, high=16.0, orig_len=131072, theta=5e5),
    dict(scaling=4, factor=16.0, mscale=1.277), dict(scaling=4, factor=4.0, orig_len=100),
    dict(scaling=4, factor=4.0, orig_len=40), dict(theta=1e6)])
@pytest.mark.parametrize("pos0", [0, 131071, 999999, FAR])
def test_scaling_and_far_positions(cuda, over, pos0):
    rp = lg.lg_default_rope_params(64, **over)
    _check(_case("f32", 64, 4, 2, [3, 7], [5, 2], cuda, pos0=pos0), rp, "f32")


def test_quarter_turns(cuda):
    """every eighth of a turn and the positions around it"""
    rp = lg.lg_default_rope_params(64, theta=1e9, rot=16)
    case = _case("f32", 64, 2, 2, [0], [3000], cuda)
    _check(case, rp, "f32")


@pytest.mark.parametrize("H_q,H_kv", [(1, 1), (5, 5), (64, 8), (7, 1)])
@pytest.mark.parametrize("ms", [[1], [1, 1, 1, 1, 1], [700, 1, 0, 0, 63], [0, 0, 2]])
def test_heads_and_ragged_chunks(cuda, H_q, H_kv, ms):
    rp = lg.lg_default_rope_params(128)
    held = [3 * i for i in range(len(ms))]
    _check(_case("bf16", 128, H_q, H_kv, held, ms, cuda, seed=H_q), rp, "bf16")


@pytest.mark.parametrize("policy", ["h2o", "streaming"])
def test_comparator_rows(cuda, policy):
    rp = lg.lg_default_rope_params(128, rot=64)
    _check(_case("bf16", 128, 8, 2, [5, 0], [3, 90], cuda, policy=policy, pos0=1000), rp, "bf16")


def test_many_sequences(cuda):
    rng = np.random.default_rng(5)
    ms = [int(x) for x in rng.integers(0, 4, 1500)]
    rp = lg.lg_default_rope_params(64)
    _check(_case("bf16", 64, 2, 2, [1] * 1500, ms, cuda), rp, "bf16")


def test_queries_in_place_and_keys_alone(cuda):
    for rot in (128, 32):
        rp = lg.lg_default_rope_params(128, rot=rot)
        case = _case("bf16", 128, 8, 2, [4], [70], cuda, packed=False)
        _check(case, rp, "bf16", q_out=case[2])
    cache, ch, q, kn, vn, pos, off = _case("bf16", 128, 8, 2, [4], [70], cuda)
    lg.lg_begin_chunk(cache, ch)
    lg.lg_rope_append(cache, ch, 0, None, kn, vn, pos, rp, None, lg.lg_default_params())
    assert lg.lg_read_device_status(cache) == 0
    _close(_np(cache.k[0, :, 4:74].transpose(0, 1)), _np(kn)[:70], np.arange(4, 74), rp, "bf16", "k")


def test_one_token_is_what_lg_append_writes(cuda):
    """position 0 turns nothing: the cache, sketches and lengths of lg_begin_step + lg_append"""
    a = _case("bf16", 128, 8, 2, [9, 4], [1, 1], cuda)
    b = _case("bf16", 128, 8, 2, [9, 4], [1, 1], cuda)
    p = lg.lg_default_params()
    cache, ch, q, kn, vn, pos, _ = a
    lg.lg_begin_chunk(cache, ch)
    lg.lg_rope_append(cache, ch, 0, q, kn, vn, torch.zeros_like(pos),
                      lg.lg_default_rope_params(128), torch.empty_like(q).contiguous(), p)
    lg.lg_begin_step(b[0])
    lg.lg_append(b[0], 0, 1, kn[:2].contiguous(), vn[:2].contiguous(), None, p)
    for x, y in ((cache.k, b[0].k), (cache.v, b[0].v), (cache.sketch, b[0].sketch),
                 (cache.len, b[0].len)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("what", ["capacity", "max_new", "T", "order", "negative"])
def test_begin_chunk_errors(cuda, what):
    cache, ch, *_ = _case("bf16", 128, 8, 2, [9, 4], [5, 6], cuda)
    off, T, mx = ch.off.clone(), ch.T, ch.max_new
    if what == "capacity":
        cache.len[1] = 6            # its capacity is 11
    elif what == "max_new":
        mx = 5
    elif what == "T":
        T = 10
    elif what == "order":
        off[1] = 12
    else:
        off[0] = -1
    lens = cache.lengths()
    lg.lg_begin_chunk(cache, lg.Chunk(off, T, mx))
    assert lg.lg_read_device_status(cache) == 4
    bad = 0 if what == "negative" else 1
    assert cache.lengths()[bad] == lens[bad]
    lg.lg_begin_chunk(cache, ch)  # skipped while the status is set
    assert cache.lengths()[bad] == lens[bad]


def test_rows_without_a_slot_are_left_out(cuda):
    """lg_rope_append without lg_begin_chunk: rows before the first slot are not written"""
    cache, ch, q, kn, vn, pos, _ = _case("bf16", 128, 8, 2, [2, 0], [5, 6], cuda)
    k0 = cache.k.clone()
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=cuda)
    lg.lg_rope_append(cache, ch, 0, q, kn, vn, pos, lg.lg_default_rope_params(128), out,
                      lg.lg_default_params())
    assert lg.lg_read_device_status(cache) == 0
    assert torch.equal(cache.k[0, :, 2:], k0[0, :, 2:]) and not torch.equal(cache.k, k0)


def test_captured_and_replayed(cuda):
    cache, ch, q, kn, vn, pos, _ = _case("bf16", 128, 8, 2, [9, 4], [3, 2], cuda)
    rp, p = lg.lg_default_rope_params(128), lg.lg_default_params()
    out = torch.empty(q.shape, dtype=q.dtype, device=cuda)
    side = torch.cuda.Stream(device=cuda)
    lg.lg_rope_append(cache, ch, 0, q, kn, vn, pos, rp, out, p)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side, capture_error_mode="thread_local"):
        lg.lg_begin_chunk(cache, ch)
        lg.lg_rope_append(cache, ch, 0, q, kn, vn, pos, rp, out, p)
    pos.add_(1000)
    g.replay()
    assert lg.lg_read_device_status(cache) == 0
    _close(_np(out)[:5], _np(q)[:5], pos.cpu().numpy()[:5], rp, "bf16", "q")
    _close(_np(cache.k[0, :, 9:12].transpose(0, 1)), _np(kn)[:3], pos.cpu().numpy()[:3], rp, "bf16",
           "k")
