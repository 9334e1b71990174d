"""Rows of a 4-bit cache: what lg_append and lg_rope_append hold, byte for byte, what lg_read_rows gives
back, and the guard's compaction of such rows."""
import math

import numpy as np
import pytest
import torch

import chunk_ref
import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


def _cache(cuda, ms, before, H_kv, d, L=1):
    ns = [n + m for n, m in zip(before, ms)]
    cap = np.array([n + 2 for n in ns], dtype=np.int32)
    seq = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
    c = lg.Cache(L, H_kv, d, "q4", seq, cap, before, cuda)
    c.k.fill_(0xaa)
    c.v.fill_(0xaa)
    return c, seq, ns


def _hard(gen, *shape):
    """rows with what quantisation can go wrong at: ties, flat groups, wide and tiny ranges"""
    x = torch.randn(shape, generator=gen)
    f = x.view(-1, shape[-1])
    f[0::7] = torch.randint(0, 16, f[0::7].shape, generator=gen) * 0.5      # codes as they are
    f[1::7] = torch.randint(0, 31, f[1::7].shape, generator=gen) * 0.25     # ties to even
    f[2::7] = 3.0                                                           # flat
    f[3::7] *= 1e30
    f[4::7] *= 1e-30
    f[5::7, ::5] += 1000.0
    return f.view(shape).bfloat16()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H_kv,batch,L", [(2, 1, 1), (2, 3, 2), (8, 65, 1), (10, 7, 3)])
def test_append_holds_the_nearest_codes(cuda, d, H_kv, batch, L):
    gen = torch.Generator().manual_seed(d + batch)
    before = [(5 * b) % 9 for b in range(batch)]
    c, seq, ns = _cache(cuda, [1] * batch, before, H_kv, d, L)
    p = lg.lg_default_params(guard_layer=L - 1)
    k, v = _hard(gen, L, batch, H_kv, d), _hard(gen, L, batch, H_kv, d)
    lg.lg_begin_step(c)
    lg.lg_append(c, 0, L, k.to(cuda), v.to(cuda), None, p)
    assert lg.lg_read_device_status(c) == 0
    for x, got in ((k, c.k.cpu()), (v, c.v.cpu())):
        want = torch.full_like(got, 0xaa)
        rows = q4_ref.packed(x)
        for b in range(batch):
            want[:, :, seq[b] + ns[b] - 1] = rows[:, b]
        assert torch.equal(got, want)
    sign = torch.signbit(v[L - 1]).view(batch, -1, 32).long()
    words = (sign << torch.arange(32)).sum(-1)
    got = c.sketch.cpu().long() & 0xffffffff
    for b in range(batch):
        assert torch.equal(got[seq[b] + ns[b] - 1], words[b])


def test_groups_that_hold_no_numbers_read_back_as_nan(cuda):
    d = 128
    c, seq, ns = _cache(cuda, [1, 1, 1, 1], [0, 0, 0, 0], 1, d)
    k = torch.zeros((1, 4, 1, d)).bfloat16()
    k[0, 0, 0, 3] = math.nan
    k[0, 1, 0, 40] = -math.inf
    k[0, 2, 0, 127] = 3e38           # a range past 2^118
    k[0, 3, 0, 70] = 3e-39           # no normal scale: held as the least value
    v = torch.randn((1, 4, 1, d)).bfloat16()
    lg.lg_begin_step(c)
    lg.lg_append(c, 0, 1, k.to(cuda), v.to(cuda), None, lg.lg_default_params())
    ko, vo = (torch.zeros((4, 1, d), dtype=torch.bfloat16, device=cuda) for _ in range(2))
    lg.lg_read_rows(c, lg.Chunk.of([1] * 4, cuda), 0, ko, vo)
    ko = ko.cpu()[:, 0].view(4, 4, 32)
    for b, bad in ((0, 0), (1, 1), (2, 3), (3, None)):
        for g in range(4):
            assert torch.isnan(ko[b, g]).all() if g == bad else (ko[b, g] == 0).all(), (b, g)
    assert torch.equal(vo.cpu()[:, 0], q4_ref.values(q4_ref.packed(v[0, :, 0])).bfloat16())


@pytest.mark.parametrize("d,rot,layout", [(128, 128, 0), (128, 64, 0), (128, 48, 1), (64, 64, 1),
                                          (64, 16, 0), (64, 32, 0)])
@pytest.mark.parametrize("ms", [[1], [3, 0, 70, 1], [513, 2]])
@pytest.mark.parametrize("packed", [True, False])
def test_rope_append(cuda, d, rot, layout, ms, packed):
    """queries as the 16-bit cache's call gives them; keys as that call's rows quantised; values too"""
    H_q, H_kv, T = 6, 2, sum(ms) + 2
    gen = torch.Generator().manual_seed(T + d)
    before = [(3 * b + 1) % 5 for b in range(len(ms))]
    c, seq, ns = _cache(cuda, ms, before, H_kv, d, 2)
    wide = lg.Cache(2, H_kv, d, "bf16", seq, [n + 2 for n in ns], before, cuda)
    x = torch.randn((T, H_q + 2 * H_kv, d), generator=gen).bfloat16().to(cuda)
    q, k, v = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pos = torch.randint(0, 1 << 20, (T,), generator=gen).int().to(cuda)
    rope = lg.lg_default_rope_params(d, rot=rot, layout=layout, mscale=1.25)
    p = lg.lg_default_params(guard_layer=1)
    ch = lg.Chunk.of(ms, cuda)
    ch = lg.Chunk(ch.off, T, ch.max_new)
    outs = []
    for cache in (wide, c):
        lg.lg_begin_chunk(cache, ch)
        out = torch.full((T, H_q, d), 7.0, dtype=torch.bfloat16, device=cuda)
        lg.lg_rope_append(cache, ch, 1, q, k, v, pos, rope, out, p)
        assert lg.lg_read_device_status(cache) == 0
        outs.append(out.cpu())
    n = sum(ms)
    # the same angles and one rounding at the end; fp32 steps may differ by an ulp before it
    diff = (outs[0][:n].float() - outs[1][:n].float()).abs()
    assert (diff <= 2.0 ** -7 * outs[0][:n].float().abs() + 2.0 ** -20).all()
    assert (diff > 0).sum() <= 2 + 1e-3 * diff.numel()
    assert (outs[1][n:] == 7.0).all()
    kc, vc, wk, wv = c.k.cpu(), c.v.cpu(), wide.k.cpu(), wide.v.cpu()
    live = torch.zeros(kc.shape[2], dtype=torch.bool)
    for b, m in enumerate(ms):
        r = slice(seq[b] + before[b], seq[b] + ns[b])
        live[r] = True
        assert torch.equal(vc[1, :, r], q4_ref.packed(wv[1, :, r]))
        got, want = q4_ref.parts(kc[1, :, r]), q4_ref.parts(q4_ref.packed(wk[1, :, r]))
        # an element that differs by a rounding may take the next code, a group's parameters the next
        # bf16 number
        off = (got[0] - want[0]).abs()
        assert (off <= 1).all() and (off > 0).sum() <= 2 + 1e-3 * off.numel()
        for i in (1, 2):
            assert ((got[i] - want[i]).abs() <= 2.0 ** -7 * want[i].abs()).all()
        assert torch.equal(c.sketch[r].cpu(), wide.sketch[r].cpu())
    for x in (kc, vc):
        assert (x[1, :, ~live] == 0xaa).all() and (x[0] == 0xaa).all()
    ko, vo = (torch.full((T, H_kv, d), 7.0, dtype=torch.bfloat16, device=cuda) for _ in range(2))
    lg.lg_read_rows(c, ch, 1, ko, vo)
    rows = torch.cat([torch.arange(seq[b] + before[b], seq[b] + ns[b]) for b in range(len(ms))])
    for got, x in ((ko.cpu(), kc), (vo.cpu(), vc)):
        assert torch.equal(got[:n], q4_ref.values(x[1][:, rows]).float().bfloat16().transpose(0, 1))
        assert (got[n:] == 7.0).all()
    # queries rotated in place give the same
    if not packed:
        lg.lg_rope_append(c, ch, 1, q, k, v, pos, rope, q, p)
        assert torch.equal(q[:n].cpu(), outs[1][:n])


def test_keys_alone_and_other_streams(cuda):
    c, seq, ns = _cache(cuda, [4, 2], [0, 3], 2, 64)
    d, T = 64, 6
    k, v = (torch.randn((T, 2, d), device=cuda).bfloat16() for _ in range(2))
    ch, pos = lg.Chunk.of([4, 2], cuda), torch.zeros(T, dtype=torch.int32, device=cuda)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        lg.lg_begin_chunk(c, ch)
        lg.lg_rope_append(c, ch, 0, None, k, v, pos, lg.lg_default_rope_params(d), None,
                          lg.lg_default_params())
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        lg.lg_read_rows(c, ch, 0, ko, vo)
    st.synchronize()
    # position zero turns nothing
    assert torch.equal(ko.cpu(), q4_ref.values(q4_ref.packed(k.cpu())).float().bfloat16())
    assert torch.equal(vo.cpu(), q4_ref.values(q4_ref.packed(v.cpu())).float().bfloat16())


@pytest.mark.parametrize("d", [64, 128])
def test_prune_moves_rows_of_four_bits(cuda, d):
    """a budget cut keeps the rows that it keeps of a 16-bit cache, byte for byte in their new slots"""
    L, H_kv, ns = 2, 4, [700, 300, 1, 900]
    cap = np.array([n + 1 for n in ns], dtype=np.int32)
    seq = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
    c = lg.Cache(L, H_kv, d, "q4", seq, cap, ns, cuda)
    c.k.random_(0, 256)
    c.v.random_(0, 256)
    c.sketch.random_()
    before = [x.cpu().clone() for x in (c.k, c.v, c.sketch)]
    budget = torch.tensor([256, 400, 256, 333], dtype=torch.int32, device=cuda)
    kept = torch.zeros((4, 1000), dtype=torch.int32, device=cuda)
    count = torch.zeros(4, dtype=torch.int32, device=cuda)
    lg.lg_prune_compact(c, None, None, None, budget, lg.lg_default_params(), kept, count, 1000, 1000)
    assert lg.lg_read_device_status(c) == 0
    lens, count, kept = c.lengths(), count.cpu().tolist(), kept.cpu()
    assert count[1] == count[2] == -1 and count[0] > 0 and count[3] > 0
    for b, n in enumerate(ns):
        idx = kept[b, :count[b]].long() if count[b] >= 0 else torch.arange(n)
        assert lens[b] == len(idx)
        o = int(seq[b])
        for x, was in zip((c.k, c.v), before):
            assert torch.equal(x.cpu()[:, :, o:o + len(idx)], was[:, :, o + idx])
        assert torch.equal(c.sketch.cpu()[o:o + len(idx)], before[2][o + idx])
