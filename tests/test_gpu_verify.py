"""lg_verify_draft against 64 bits, and lg_end_chunk."""
import math

import numpy as np
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu


def _case(ms, V, dtype, certain, seed, noise=0.7, hot=True):
    gen = torch.Generator().manual_seed(seed)
    T = sum(ms)
    x = torch.randn((T, V), generator=gen) * 2
    if hot:
        x.scatter_add_(1, torch.randint(0, V, (T, 3), generator=gen), torch.full((T, 3), 7.0))
    y = x + noise * torch.randn((T, V), generator=gen)
    x = x if dtype == "f32" else x.bfloat16()
    q = y.softmax(-1)
    q = q if dtype == "f32" else q.bfloat16()
    drawn = torch.multinomial(q.float(), 1, generator=gen)[:, 0]
    tokens = torch.cat([drawn[-1:], drawn[:-1]]).int()
    temp = torch.rand(len(ms), generator=gen) + 0.5
    temp[2::3] = 0.0
    return (x, ms, tokens, None if certain else q, temp, torch.rand(T, generator=gen),
            torch.rand(len(ms), generator=gen))


def _run(cuda, x, ms, tokens, draft, temp, u, r, pad=2):
    """(picked, accepted); rows behind the last sequence are not touched"""
    T = sum(ms) + pad

    def rows(a):  # the same rows at an odd stride, rows of NaN behind them
        if a is None:
            return None
        buf = torch.full((T, a.shape[1] + 3), math.nan, dtype=a.dtype, device=cuda)
        buf[:sum(ms), 1:1 + a.shape[1]] = a.to(cuda)
        return buf[:, 1:1 + a.shape[1]]

    def long(a, fill):
        return torch.cat([a, torch.full((pad,), fill, dtype=a.dtype)]).to(cuda)

    ch = lg.Chunk.of(ms, cuda)
    ch = lg.Chunk(ch.off, T, ch.max_new)
    xs, status = rows(x), torch.zeros(1, dtype=torch.int32, device=cuda)
    picked = torch.full((T,), 77, dtype=torch.int32, device=cuda)
    accepted = torch.full((len(ms),), 77, dtype=torch.int32, device=cuda)
    ws = torch.full((lg.lg_verify_workspace_size(xs, ch),), 0xff, dtype=torch.uint8, device=cuda)
    lg.lg_verify_draft(xs, ch, long(tokens, 5), rows(draft), None if temp is None else temp.to(cuda),
                       long(u, 0.5), r.to(cuda), picked, accepted, ws, status)
    assert status.item() == 0
    picked = picked.cpu().tolist()
    assert picked[sum(ms):] == [77] * pad
    return picked[:sum(ms)], accepted.cpu().tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("V", [1, 2, 7, 33, 1000, 4097, 32003])
def test_against_64_bits(cuda, dtype, certain, V):
    for seed, ms in ((1, [1]), (2, [4]), (3, [3, 1, 0, 6, 2, 5, 1]), (4, [2] * 40), (5, [18, 20])):
        if V > 5000 and len(ms) > 7:
            continue
        c = _case(ms, V, dtype, certain, seed)
        assert _run(cuda, *c) == q4_ref.verify(*c)


def test_a_large_vocabulary(cuda):
    for dtype in ("bf16", "f32"):
        c = _case([5, 1, 3], 151937, dtype, False, 9)
        assert _run(cuda, *c) == q4_ref.verify(*c)


def test_what_is_masked_or_infinite(cuda):
    V, ms = 300, [3, 2, 2, 2, 2, 1]
    x, ms, tokens, q, temp, u, r = _case(ms, V, "f32", False, 5)
    temp[:] = 1.0
    temp[1] = 0.0
    x[0, 10:] = -math.inf
    x[1, ::2] = math.nan
    x[3] = 0.25                                  # ties: the lowest
    x[5], x[6] = -math.inf, -math.inf            # nothing left: the draft falls, no token
    x[7, 20], x[7, 31] = math.inf, math.inf      # the mass is shared
    x[9, :5] = math.nan
    tokens[10] = -3                              # a draft that is no token
    q[2, 4:9] = math.nan
    q[0, 3] = -1.0
    for k in range(20):
        g = torch.Generator().manual_seed(k)
        u, r = torch.rand(u.shape, generator=g), torch.rand(r.shape, generator=g)
        assert _run(cuda, x, ms, tokens, q, temp, u, r) == \
            q4_ref.verify(x, ms, tokens, q, temp, u, r)


@pytest.mark.parametrize("r", [0.0, 1.0, 2.0, -1.0, math.nan, 1 - 2.0 ** -24])
def test_borders_of_the_random_numbers(cuda, r):
    V, ms = 200, [1, 3]
    x, ms, tokens, q, temp, u, _ = _case(ms, V, "f32", False, 8)
    x[:, 0] = x[:, V - 1] = -math.inf
    rr = torch.full((2,), r)
    got, want = _run(cuda, x, ms, tokens, q, None, u, rr), q4_ref.verify(x, ms, tokens, q, None, u, rr)
    if math.isnan(r) or r <= 0:
        assert got == want
    else:  # next to the end the last tokens' own rounding decides: any of the lowest mass there is
        assert got[1] == want[1]
        for a, b in zip(got[0], want[0]):
            assert a == b or b >= V - 8 and a >= V - 8


@pytest.mark.parametrize("batch", [1, 3, 40, 160])  # clusters of sixteen CTAs to one
def test_a_number_on_a_bound(cuda, batch):
    """equal tokens, every sum exact: r = j / n is the bound below token j, which it belongs to"""
    n = 4096
    j = torch.randint(0, n, (batch,), generator=torch.Generator().manual_seed(3))
    x = torch.full((batch, n), 0.25)
    c = (x, [1] * batch, torch.zeros(batch, dtype=torch.int32), None, None, torch.zeros(batch))
    picked, _ = _run(cuda, *c, j / n)
    assert picked == j.tolist()
    # of a draft's row what it lacks: the upper half (its first token falls, 0.75 q = 1.5 p)
    m = 2 * batch
    q = torch.zeros((m, n))
    q[:, :n // 2] = 2 / n
    c = (torch.full((m, n), 0.25), [2] * batch, torch.full((m,), 7, dtype=torch.int32), q, None,
         torch.full((m,), 0.75))
    j = j // 2
    picked, accepted = _run(cuda, *c, j / (n // 2))
    assert accepted == [0] * batch
    assert picked[0::2] == (n // 2 + j).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("batch", [2, 40, 160])
def test_numbers_next_to_a_bound(cuda, dtype, certain, batch):
    """r the 32-bit number before or after a bound of 64-bit sums, some 2^-32 from it: fp32 masses
    are some 2^-28 off"""
    V = 9001
    x, ms, tokens, q, _, u, _ = _case([2] * batch, V, dtype, certain, 21, hot=False)
    u[:] = 1 - 2 ** -24  # most drafts fall
    p = x.double().softmax(-1)
    r = torch.zeros(batch)
    for b in range(batch):
        first = not (u[2 * b].double() * (1 if certain else q[2 * b, tokens[2 * b + 1]].double())
                     < p[2 * b, tokens[2 * b + 1]])
        w = p[2 * b] if first else p[2 * b + 1]
        if first and certain:
            w = w.clone()
            w[tokens[2 * b + 1]] = 0
        elif first:
            w = (w - q[2 * b].double()).clamp(min=0)
        cum = w.cumsum(0) / w.sum()
        bound = cum[int((cum < 2 ** -7).sum()) + b % 5]
        at = np.float32(bound.item())
        r[b] = float(np.nextafter(at, np.float32(b % 2)))
    c = (x, ms, tokens, q, None, u, r)
    assert _run(cuda, *c) == q4_ref.verify(*c)


def test_temperatures_out_of_range(cuda):
    x, ms, tokens, q, _, u, r = _case([2, 2, 2, 2], 500, "f32", False, 4)
    temp = torch.tensor([-1.0, math.nan, math.inf, 1e-35])
    assert _run(cuda, x, ms, tokens, q, temp, u, r) == q4_ref.verify(x, ms, tokens, q, temp, u, r)


def test_the_same_distribution_leaves_every_draft(cuda):
    """p = q up to rounding: u q < p for u away from one, and with nothing left the token is p's"""
    V, ms = 64, [5]
    x = torch.randn((5, V))
    q = x.double().softmax(-1).float()
    tokens = torch.randint(0, V, (5,)).int()
    got = _run(cuda, x, ms, tokens, q, None, torch.full((5,), 0.999), torch.full((1,), 0.5))
    assert got[1] == [4]
    # a draft that claims more than it may (q = 2): w is empty, and p takes its place
    got = _run(cuda, x, ms, tokens, torch.full((5, V), 2.0), None, torch.full((5,), 0.999),
               torch.full((1,), 0.5))
    p = x[0].double().softmax(-1).cumsum(0)
    assert got == ([int((p > 0.5).nonzero()[0])] + [-1] * 4, [0])


def test_tokens_follow_the_target(cuda):
    """20000 sequences of one draft each: the first token's frequencies are the target's, whatever the
    draft's (each frequency within 5 of its deviations)"""
    V, B = 8, 20000
    g = torch.Generator().manual_seed(0)
    p = torch.tensor([0.3, 0.05, 0.2, 0.0, 0.15, 0.1, 0.12, 0.08])
    q = torch.tensor([0.05, 0.3, 0.1, 0.2, 0.05, 0.1, 0.1, 0.1])
    x = p.log()[None].repeat(2 * B, 1)
    drawn = torch.multinomial(q, 2 * B, replacement=True, generator=g).int()
    picked, _ = _run(cuda, x, [2] * B, drawn, q[None].repeat(2 * B, 1), None,
                     torch.rand(2 * B, generator=g), torch.rand(B, generator=g), pad=0)
    f = np.bincount(np.array(picked)[0::2], minlength=V) / B
    for i in range(V):
        assert abs(f[i] - p[i]) <= 5 * math.sqrt(p[i] * (1 - p[i]) / B) + 1e-12


def test_bits_do_not_depend_on_the_batch(cuda):
    x, ms, tokens, q, temp, u, r = _case([3, 2, 4], 9001, "bf16", False, 12)
    whole = _run(cuda, x, ms, tokens, q, temp, u, r)[0]
    t = 0
    for b, m in enumerate(ms):
        s = slice(t, t + m)
        assert _run(cuda, x[s], [m], tokens[s], q[s], temp[b:b + 1], u[s], r[b:b + 1])[0] == whole[s]
        t += m


def test_status_and_captured_calls(cuda):
    x, ms, tokens, q, temp, u, r = (a.to(cuda) if torch.is_tensor(a) else a
                                    for a in _case([3, 2], 700, "bf16", False, 3))
    ch = lg.Chunk.of(ms, cuda)
    status = torch.zeros(1, dtype=torch.int32, device=cuda)
    picked, accepted = torch.empty(5, dtype=torch.int32, device=cuda), \
        torch.empty(2, dtype=torch.int32, device=cuda)
    ws = torch.empty(lg.lg_verify_workspace_size(x, ch), dtype=torch.uint8, device=cuda)
    call = lambda c=ch: lg.lg_verify_draft(x, c, tokens, q, temp, u, r, picked, accepted, ws, status)
    call()
    want = picked.clone(), accepted.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    picked.fill_(9)
    g.replay()
    assert torch.equal(picked, want[0]) and torch.equal(accepted, want[1])
    call(lg.Chunk(ch.off, 5, 2))          # a sequence of more rows than announced
    assert status.item() == 4
    picked.fill_(9)
    call()                                # skipped from now on
    assert (picked == 9).all()


def test_a_step_of_no_rows(cuda):
    """every sequence rests: nothing is read, nothing stands"""
    x = torch.full((1, 50), math.nan, device=cuda)
    ch = lg.Chunk.of([0, 0, 0], cuda)
    z = torch.zeros(3, device=cuda)
    picked = torch.full((1,), 9, dtype=torch.int32, device=cuda)
    acc = torch.full((3,), 9, dtype=torch.int32, device=cuda)
    ws = torch.empty(lg.lg_verify_workspace_size(x, ch), dtype=torch.uint8, device=cuda)
    lg.lg_verify_draft(x, ch, picked.clone(), None, None, z, z, picked, acc, ws)
    assert acc.tolist() == [0, 0, 0] and picked.tolist() == [9]


def test_end_chunk(cuda):
    ns, ms = [10, 7, 5, 3], [4, 1, 0, 3]
    c = lg.Cache(1, 2, 64, "bf16", [0, 20, 40, 60], [20] * 4, ns, cuda)
    ch = lg.Chunk.of(ms, cuda)
    acc = torch.tensor([1, 0, 0, 2], dtype=torch.int32, device=cuda)
    lg.lg_end_chunk(c, ch, acc)
    assert lg.lg_read_device_status(c) == 0 and c.lengths().tolist() == [8, 7, 5, 3]
    c = lg.Cache(1, 2, 64, "bf16", [0, 20, 40, 60], [20] * 4, ns, cuda)
    acc[2] = -7                                       # of a sequence that had no rows
    lg.lg_end_chunk(c, ch, acc)
    assert lg.lg_read_device_status(c) == 0 and c.lengths().tolist() == [8, 7, 5, 3]
    for bad in ([4, 0, 0, 2], [-1, 0, 0, 2], [1, 1, 0, 2]):
        c = lg.Cache(1, 2, 64, "bf16", [0, 20, 40, 60], [20] * 4, ns, cuda)
        lg.lg_end_chunk(c, ch, torch.tensor(bad, dtype=torch.int32, device=cuda))
        assert lg.lg_read_device_status(c) == 4
