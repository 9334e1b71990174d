"""Decode steps over a 4-bit cache as a user makes them: drafted tokens that join the cache, attend, are
verified and leave it again; the guard's steps with a prune; both captured into a graph."""
import numpy as np
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu

L, H_KV, G, D, V = 2, 2, 4, 128, 1003
H_Q = H_KV * G
LENS = [150, 33, 1]


class Model:
    """random weights; what a layer projects depends on its attention output"""

    def __init__(self, cuda):
        g = torch.Generator(device=cuda)
        g.manual_seed(3)
        n = H_Q * D
        r = lambda *s: torch.randn(s, generator=g, device=cuda)
        self.emb = r(V, n).bfloat16()
        self.w = [r(n, (H_Q + 2 * H_KV) * D).mul_(n ** -0.5).bfloat16() for _ in range(L)]
        self.head = r(n, V).mul_(4 * n ** -0.5).bfloat16()
        self.rope, self.p = lg.lg_default_rope_params(D), lg.lg_default_params()

    def layers(self, cache, ch, rows, pos, ws, max_len):
        x, T = self.emb[rows.long()], rows.shape[0]
        for l in range(L):
            qkv = (x @ self.w[l]).view(T, H_Q + 2 * H_KV, D)
            q = torch.empty((T, H_Q, D), dtype=x.dtype, device=x.device)
            o = torch.empty_like(q)
            lg.lg_rope_append(cache, ch, l, qkv[:, :H_Q], qkv[:, H_Q:H_Q + H_KV], qkv[:, H_Q + H_KV:],
                              pos, self.rope, q, self.p)
            lg.lg_chunk_attend(cache, ch, l, q, H_Q, D ** -0.5, 0, 0, o, max_len, ws)
            x = x + o.view(T, -1)
        return (x @ self.head).float()


def _cache(cuda, dtype, cap=260):
    seq = np.arange(len(LENS)) * cap
    return lg.Cache(L, H_KV, D, dtype, seq, [cap] * len(LENS), [0] * len(LENS), cuda), seq


def _ws(cache, ch, cuda):
    return torch.empty(lg.lg_chunk_workspace_size(cache, ch, H_Q, 260), dtype=torch.uint8, device=cuda)


@pytest.mark.parametrize("dtype", ["q4", "bf16"])
def test_drafted_steps(cuda, dtype):
    """prompts, then steps of up to five drafts: picks as defined on the step's own logits, lengths, the
    history, and rows of the first layer that are those of the tokens that stood, in order"""
    model, rng = Model(cuda), np.random.default_rng(5)
    cache, seq = _cache(cuda, dtype)
    ids = [list(rng.integers(0, V, n)) for n in LENS]          # tokens in the cache
    ch = lg.Chunk.of(LENS, cuda)
    lg.lg_begin_chunk(cache, ch)
    pos = torch.as_tensor(np.concatenate([np.arange(n) for n in LENS]).astype(np.int32), device=cuda)
    model.layers(cache, ch, torch.as_tensor(np.concatenate(ids), device=cuda), pos, _ws(cache, ch, cuda),
                 260)
    head = [int(x) for x in rng.integers(0, V, 3)]             # each sequence's next token
    seen = torch.zeros((3, (V + 31) // 32), dtype=torch.int32, device=cuda)
    counts = torch.zeros((3, V), dtype=torch.int32, device=cuda)
    want_counts = np.zeros((3, V), dtype=np.int64)
    temp = torch.tensor([0.8, 0.0, 1.1], device=cuda)
    accepted_any = 0
    for step in range(8):
        ks = [int(k) for k in rng.integers(0, 6, 3)]
        if step == 3:
            ks[1] = -1                                          # this sequence rests: no rows
        ms = [k + 1 for k in ks]
        rows, poss = [], []
        for b in range(3):
            for j in range(ms[b]):
                rows.append(head[b] if j == 0 else int(rng.integers(0, V)))
                poss.append(len(ids[b]) + j)
        ch, T = lg.Chunk.of(ms, cuda), len(rows)
        tokens = torch.tensor(rows, dtype=torch.int32, device=cuda)
        pos = torch.tensor(poss, dtype=torch.int32, device=cuda)
        lg.lg_begin_chunk(cache, ch)
        logits = model.layers(cache, ch, tokens, pos, _ws(cache, ch, cuda), 260)
        if step % 2:  # drafts that the model likes, so that some stand: the model's own choices
            off = np.concatenate([[0], np.cumsum(ms)])
            for b in range(3):
                for t in range(off[b], off[b + 1] - 1):
                    tokens[t + 1] = int(logits[t].argmax())
        u, r = (torch.rand(n, device=cuda) for n in (T, 3))
        draft = None if step % 3 else torch.full((T, V), 0.3 / V, device=cuda)
        picked = torch.empty(T, dtype=torch.int32, device=cuda)
        acc = torch.empty(3, dtype=torch.int32, device=cuda)
        vws = torch.empty(lg.lg_verify_workspace_size(logits, ch), dtype=torch.uint8, device=cuda)
        lg.lg_verify_draft(logits, ch, tokens, draft, temp, u, r, picked, acc, vws, cache.status)
        lg.lg_end_chunk(cache, ch, acc)
        lg.lg_count_tokens(picked, ch.off, V, 1, seen, counts, cache.status)
        assert lg.lg_read_device_status(cache) == 0
        want = q4_ref.verify(logits.cpu(), ms, tokens.cpu(), None if draft is None else draft.cpu(),
                             temp.cpu(), u.cpu(), r.cpu())
        assert (picked.cpu().tolist(), acc.cpu().tolist()) == want
        # the rows that were appended are the first tokens as they were asked for (drafts swapped in
        # above came after the append: they only test the verification)
        t = 0
        for b in range(3):
            if ms[b]:
                a = want[1][b]
                accepted_any += a
                ids[b] += [rows[t]] + rows[t + 1:t + 1 + a]
                head[b] = want[0][t + a]
                for x in want[0][t:t + a + 1]:
                    want_counts[b, x] += 1
            t += ms[b]
        assert cache.lengths().tolist() == [len(x) for x in ids]
    assert accepted_any > 5
    assert np.array_equal(counts.cpu().numpy(), want_counts)
    # layer 0's rows depend on tokens and positions alone: one chunk of all that stood
    fresh, _ = _cache(cuda, dtype)
    ns = [len(x) for x in ids]
    ch = lg.Chunk.of(ns, cuda)
    lg.lg_begin_chunk(fresh, ch)
    rows = torch.as_tensor(np.concatenate(ids), device=cuda)
    qkv = (model.emb[rows.long()] @ model.w[0]).view(-1, H_Q + 2 * H_KV, D)
    pos = torch.as_tensor(np.concatenate([np.arange(n) for n in ns]).astype(np.int32), device=cuda)
    lg.lg_rope_append(fresh, ch, 0, None, qkv[:, H_Q:H_Q + H_KV], qkv[:, H_Q + H_KV:], pos, model.rope,
                      None, model.p)
    for b, n in enumerate(ns):
        o = int(seq[b])
        for x, y in ((cache.k, fresh.k), (cache.v, fresh.v)):
            a, e = x[0, :, o:o + n], y[0, :, o:o + n]
            if dtype == "q4":  # (matrix products of other shapes may round a projection otherwise)
                a, e = q4_ref.values(a.cpu()), q4_ref.values(e.cpu())
            d = (a.double() - e.double()).abs().amax(-1)
            s = e.double().abs().amax(-1)
            assert (d <= (0.15 if dtype == "q4" else 2.0 ** -6) * s).all()


def test_guarded_steps_and_a_prune(cuda):
    """Guard over four bits beside Guard over the same rows in bf16: the same decisions, rows and sketches,
    statistics within the rounding of the values"""
    cap, n0 = 700, [600, 420]
    seq = np.array([0, cap])
    p = lg.lg_default_params()
    q4 = lg.Cache(L, H_KV, D, "q4", seq, [cap] * 2, [0, 0], cuda)
    wide = lg.Cache(L, H_KV, D, "bf16", seq, [cap] * 2, [0, 0], cuda)
    g = torch.Generator(device=cuda)
    g.manual_seed(9)
    T = sum(n0)
    ch, pos = lg.Chunk.of(n0, cuda), torch.zeros(T, dtype=torch.int32, device=cuda)
    rope = lg.lg_default_rope_params(D)
    for c in (q4, wide):
        lg.lg_begin_chunk(c, ch)
    for l in range(L):
        k, v = (torch.randn((T, H_KV, D), generator=g, device=cuda).bfloat16() for _ in range(2))
        v[400:600] = v[360:400].repeat(5, 1, 1)                 # a loop of period 40 ends sequence 0
        lg.lg_rope_append(q4, ch, l, None, k, v, pos, rope, None, p)
        lg.lg_rope_append(wide, ch, l, None, k, v, pos, rope, None, p)
    for l in range(L):                                          # ... and the values that four bits hold
        ko, vo = (torch.empty((T, H_KV, D), dtype=torch.bfloat16, device=cuda) for _ in range(2))
        lg.lg_read_rows(q4, ch, l, ko, vo)
        for b, o in enumerate(seq):
            s = slice(sum(n0[:b]), sum(n0[:b + 1]))
            wide.k[l, :, o:o + n0[b]] = ko[s].transpose(0, 1)
            wide.v[l, :, o:o + n0[b]] = vo[s].transpose(0, 1)
    assert torch.equal(q4.sketch, wide.sketch)
    guards = [lg.Guard(c, H_Q, p, max_len=cap) for c in (q4, wide)]
    budget = torch.tensor([512, 512], dtype=torch.int32, device=cuda)
    for step in range(4):
        q = torch.randn((L, 2, H_Q, D), generator=g, device=cuda).bfloat16()
        kn, vn = (torch.randn((L, 2, H_KV, D), generator=g, device=cuda).bfloat16() for _ in range(2))
        res = []
        for gd in guards:
            gd.step(q, kn, vn, budget)
            res.append(gd.results())
        a, b = res
        for name in ("flags", "spans", "len", "kept_count", "state"):
            assert np.array_equal(a[name], b[name]), name
        for i, n in enumerate(a["kept_count"]):
            assert np.array_equal(a["kept_idx"][i, :max(n, 0)], b["kept_idx"][i, :max(n, 0)])
        assert np.allclose(a["stats"], b["stats"], rtol=2e-2, atol=2e-2)
        assert np.allclose(a["out"], b["out"], rtol=0.1, atol=0.02)
        if step == 0:
            assert a["kept_count"][0] > 0                       # over its budget: cut
            moved = True
    assert moved and torch.equal(q4.sketch[:512], wide.sketch[:512])


def test_a_captured_step(cuda):
    """begin, append, attention, verification and end in one graph, replayed: as the calls one by one"""
    gen = torch.Generator().manual_seed(2)
    cap, n0, ms = 400, [100, 64, 7], [3, 1, 4]
    seq = np.arange(3) * cap
    T = sum(ms)
    rope, p = lg.lg_default_rope_params(D), lg.lg_default_params()
    ch = lg.Chunk.of(ms, cuda)
    x = torch.randn((T, H_Q + 2 * H_KV, D), generator=gen).bfloat16().to(cuda)
    pos = torch.arange(T, dtype=torch.int32, device=cuda)
    logits, u, r = torch.randn((T, V), generator=gen).to(cuda), torch.rand(T).to(cuda), torch.rand(3).to(cuda)
    tokens = torch.randint(0, V, (T,), generator=gen).int().to(cuda)
    start = torch.randint(0, 120, (1, H_KV, 3 * cap, D // 2 + 16), generator=gen).to(torch.uint8).to(cuda)

    def run(steps, graph):
        c = lg.Cache(1, H_KV, D, "q4", seq, [cap] * 3, n0, cuda, "loopguard", start.clone(), start.clone())
        q, o = (torch.empty((T, H_Q, D), dtype=torch.bfloat16, device=cuda) for _ in range(2))
        ws = torch.empty(lg.lg_chunk_workspace_size(c, ch, H_Q, cap), dtype=torch.uint8, device=cuda)
        vws = torch.empty(lg.lg_verify_workspace_size(logits, ch), dtype=torch.uint8, device=cuda)
        picked = torch.empty(T, dtype=torch.int32, device=cuda)
        acc = torch.empty(3, dtype=torch.int32, device=cuda)

        def step():
            lg.lg_begin_chunk(c, ch)
            lg.lg_rope_append(c, ch, 0, x[:, :H_Q], x[:, H_Q:H_Q + H_KV], x[:, H_Q + H_KV:], pos, rope, q, p)
            lg.lg_chunk_attend(c, ch, 0, q, H_Q, D ** -0.5, 0, 0, o, cap, ws)
            lg.lg_verify_draft(logits, ch, tokens, None, None, u, r, picked, acc, vws, c.status)
            lg.lg_end_chunk(c, ch, acc)

        if graph:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for _ in range(steps):
                g.replay()
        else:
            for _ in range(steps):
                step()
        assert lg.lg_read_device_status(c) == 0
        return c.k, c.v, c.sketch, o, picked, acc, c.len

    for a, b in zip(run(5, False), run(5, True)):
        assert torch.equal(a, b)
