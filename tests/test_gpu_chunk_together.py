"""The calls of include/lg_chunk.h as a model step makes them, one after another on the guard's
cache: a prompt in chunks, then guarded decode steps whose tokens come from the step's logits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import chunk_ref
from paper_2604_10044_gb300 import lg

pytestmark = pytest.mark.gpu

L, H_KV, G, D, V = 2, 2, 4, 128, 4001
H_Q = H_KV * G


class Model:
    """random weights and tied activations: what a layer projects depends on its attention output,
    so a wrong row anywhere changes the tokens that follow"""

    def __init__(self, cuda, dtype):
        g = torch.Generator(device=cuda)
        g.manual_seed(3)
        dt = chunk_ref.tdtype(dtype)
        n = H_Q * D
        self.emb = torch.randn((V, n), generator=g, device=cuda).to(dt)
        self.w = [torch.randn((n, (H_Q + 2 * H_KV) * D), generator=g, device=cuda).mul_(n ** -0.5).to(dt)
                  for _ in range(L)]
        self.head = torch.randn((n, V), generator=g, device=cuda).mul_(n ** -0.5).to(dt)


def _chunk(model, cache, rows, ms, pos, rope, p, window, sink, ws, max_len):
    """one pass of `rows` (token ids of every sequence, one after another); the last layer's output"""
    ch = lg.Chunk.of(ms, cache.device)
    lg.lg_begin_chunk(cache, ch)
    x = model.emb[rows]
    T = len(rows)
    for l in range(L):
        qkv = (x @ model.w[l]).view(T, H_Q + 2 * H_KV, D)
        q = torch.empty((T, H_Q, D), dtype=x.dtype, device=x.device)
        o = torch.empty_like(q)
        lg.lg_rope_append(cache, ch, l, qkv[:, :H_Q], qkv[:, H_Q:H_Q + H_KV], qkv[:, H_Q + H_KV:],
                          pos, rope, q, p)
        lg.lg_chunk_attend(cache, ch, l, q, H_Q, D ** -0.5, window, sink, o, max_len, ws)
        x = x + o.view(T, -1)
    return x, ch


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(0, 0), (40, 4)])
def test_prompt_in_chunks_is_the_prompt(cuda, dtype, window, sink):
    """the same prompts in one chunk and in pieces of different sizes: the same cache within the
    rounding of the attention outputs that later layers' rows come from"""
    model = Model(cuda, dtype)
    lens = [150, 70, 1]
    cap = np.array([n + 4 for n in lens], dtype=np.int32)
    seq = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
    rng = np.random.default_rng(1)
    ids = [rng.integers(0, V, n) for n in lens]
    rope, p = lg.lg_default_rope_params(D), lg.lg_default_params()
    caches, last = [], []
    for cuts in ([[150], [70], [1]], [[64, 1, 85], [0, 70, 0], [0, 0, 1]],
                 [[5, 5, 140], [69, 0, 1], [1, 0, 0]]):
        cache = lg.Cache(L, H_KV, D, dtype, seq, cap, [0, 0, 0], cuda)
        done = [0, 0, 0]
        ends = {}
        for step in range(len(cuts[0])):
            ms = [c[step] for c in cuts]
            rows = np.concatenate([ids[b][done[b]:done[b] + ms[b]] for b in range(3)])
            pos = np.concatenate([np.arange(done[b], done[b] + ms[b]) for b in range(3)])
            ch = lg.Chunk.of(ms, cuda)
            ws = torch.empty(lg.lg_chunk_workspace_size(cache, ch, H_Q, 154), dtype=torch.uint8,
                             device=cuda)
            x, ch = _chunk(model, cache, torch.as_tensor(rows, device=cuda), ms,
                           torch.as_tensor(pos.astype(np.int32), device=cuda), rope, p, window, sink,
                           ws, 154)
            off = ch.off.cpu().numpy()
            for b in range(3):
                done[b] += ms[b]
                if ms[b]:
                    ends[b] = x[off[b + 1] - 1]
        assert lg.lg_read_device_status(cache) == 0
        assert (cache.lengths() == lens).all()
        caches.append(cache)
        last.append(torch.stack([ends[b] for b in range(3)]))
    # layer 0's rows do not depend on the attention; its sketches are the guard's
    for c in caches[1:]:
        for b, n in enumerate(lens):
            o = int(seq[b])
            rel = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) * 4
            for x, y in ((c.k, caches[0].k), (c.v, caches[0].v)):
                a, e = x[:, :, o:o + n].float(), y[:, :, o:o + n].float()
                assert (a - e).abs().max() <= rel * e.abs().max()
    for x in last[1:]:
        assert (x - last[0]).float().abs().max() <= 2.0 ** -5 * last[0].float().abs().max()


def test_a_guarded_decode_from_logits(cuda):
    """prompt by chunk, then single-token chunks beside lg_decode_attend on the same rows, the
    picked token and its probability read by the token-level monitor with its retained set"""
    model = Model(cuda, "bf16")
    lens, steps, budget = [90, 40], 120, 128
    cap = np.array([budget + 2] * 2, dtype=np.int32)
    seq = np.array([0, budget + 2], dtype=np.int64)
    cache = lg.Cache(L, H_KV, D, "bf16", seq, cap, [0, 0], cuda)
    rope, p = lg.lg_default_rope_params(D), lg.lg_default_params(n_anchor=8, t_min=4)
    tp = lg.lg_default_token_params()
    g = lg.Guard(cache, H_Q, p, max_len=budget + 2)
    lg.lg_state_init(cache, g.state, 0)
    tstate = torch.zeros(lg.lg_token_state_size(cache, p, tp) // 4, dtype=torch.int32, device=cuda)
    rng = np.random.default_rng(2)
    ids = [rng.integers(0, V, n) for n in lens]
    nw = (V + 31) // 32
    seen = torch.zeros((2, nw), dtype=torch.int32, device=cuda)
    counts = torch.zeros((2, V), dtype=torch.int32, device=cuda)
    rows = torch.as_tensor(np.concatenate(ids).astype(np.int32), device=cuda)
    off = torch.tensor([0, 90, 130], dtype=torch.int32, device=cuda)
    lg.lg_count_tokens(rows, off, V, 0, seen, counts, cache.status)
    pos = torch.as_tensor(np.concatenate([np.arange(n) for n in lens]).astype(np.int32), device=cuda)
    ws = torch.empty(lg.lg_chunk_workspace_size(cache, lg.Chunk.of(lens, cuda), H_Q, budget + 2),
                     dtype=torch.uint8, device=cuda)
    x, ch = _chunk(model, cache, rows.long(), lens, pos, rope, p, 0, 0, ws, budget + 2)
    x = x[[89, 129]]
    tok = torch.zeros(2, dtype=torch.int32, device=cuda)
    pm = torch.zeros(2, device=cuda)
    pen = torch.tensor([[1.0, 0.0, 0.0, 0.0], [1.2, 0.1, 0.05, 0.0]], device=cuda)
    budget_d = torch.full((2,), budget, dtype=torch.int32, device=cuda)
    kept_count = torch.full((2,), -1, dtype=torch.int32, device=cuda)
    g.kept_count.copy_(kept_count)
    at = torch.tensor(lens, dtype=torch.int32, device=cuda)
    host_seen = [set(i.tolist()) for i in ids]
    host_count = np.zeros((2, V), dtype=np.int64)
    pruned = 0
    for step in range(steps):
        logits = (x @ model.head).float() * 2.0
        lg.lg_pick_token(logits, seen, counts, pen, None, None, tok, pm, cache.status)
        lg.lg_count_tokens(tok, None, V, 1, seen, counts, cache.status)
        for b in range(2):
            s = np.zeros(V, dtype=bool)
            s[list(host_seen[b])] = True
            want, pw, _ = chunk_ref.pick(logits[b].cpu().numpy(), s, host_count[b],
                                         pen[b].tolist(), None, None)
            assert tok[b].item() == want and abs(pm[b].item() - pw) <= 1e-3 * pw
            host_seen[b].add(want)
            host_count[b, want] += 1
        x, ch = _chunk(model, cache, tok.long(), [1, 1], at, rope, p, 0, 0, ws, budget + 2)
        at += 1
        # the last layer's decode attention over the same rows, from the general call
        q = torch.randn((1, 2, H_Q, D), device=cuda).bfloat16()
        out, o2 = torch.empty_like(q), torch.empty_like(q[0])
        stats = torch.empty((1, 2, H_Q, 4), device=cuda)
        lg.lg_decode_attend(cache, L - 1, 1, q, H_Q, D ** -0.5, out, stats, 64, 0, budget + 2, g.ws)
        lg.lg_chunk_attend(cache, ch, L - 1, q[0], H_Q, D ** -0.5, 0, 0, o2, budget + 2, ws)
        assert (out[0].float() - o2.float()).abs().max() <= 2.0 ** -6 * out.float().abs().max()
        lg.lg_token_detect_prune(cache, tok, pm, g.state, budget_d, p, tp, g.flags, g.spans, None,
                                 tstate, g.kept_idx, g.kept_count, g.max_keep, g.max_len)
        assert lg.lg_read_device_status(cache) == 0
        pruned += int((g.kept_count >= 0).sum().item())
        assert (cache.lengths() <= budget).all()
    assert pruned > 0 and cache.lengths().min() > 8


FIRST = """
import torch
from paper_2604_10044_gb300 import lg
import chunk_ref
b = chunk_ref.Batch([300, 2000], [200, 2000], "bf16", H_kv=8, g=2).to_device()
b.max_len = 20000
x = torch.randn((20, 50000), device="cuda")
tok = torch.zeros(20, dtype=torch.int32, device="cuda")
pm = torch.zeros(20, device="cuda")
out = torch.full_like(b.qd, 7.0)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    lg.lg_chunk_attend(b.cache, b.chunk, 0, b.qd, b.H_q, b.d ** -0.5, 0, 0, out, b.max_len, b.ws)
    lg.lg_pick_token(x, None, None, None, None, None, tok, pm)
g.replay()
torch.cuda.synchronize()
b.check(out)
assert torch.equal(tok.long(), x.argmax(-1))
print("ok")
"""


def test_a_process_may_begin_with_captured_calls(cuda):
    """nothing that a first call sets up is forbidden while a stream is captured"""
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(here), here]))
    r = subprocess.run([sys.executable, "-c", FIRST], env=env, capture_output=True, text=True,
                       timeout=240)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr[-2000:]
