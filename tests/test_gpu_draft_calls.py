"""Calls over a 4-bit cache and of lg_verify_draft as programs make them beside one another: on a stream of
the caller's own, from several host threads, drafts of another type than the logits, a prompt's chunk in a
batch of single tokens."""
import threading

import numpy as np
import pytest
import torch

import q4_ref
from paper_2604_10044_gb300 import lg
from test_gpu_verify import _case, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("xt,qt", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("V", [33, 4097])
def test_drafts_of_another_type(cuda, xt, qt, V):
    x, ms, tokens, q, temp, u, r = _case([3, 1, 0, 6, 2], V, xt, False, 7)
    q = q.float() if qt == "f32" else q.bfloat16()
    c = (x, ms, tokens, q, temp, u, r)
    assert _run(cuda, *c) == q4_ref.verify(*c)


def _jobs(cuda, seed):
    """attention and verification with buffers of their own: (call on a stream, outputs, what they should
    hold)"""
    b = q4_ref.Batch([900, 40, 333], [5, 1, 2], seed=seed, device=cuda).to_device()
    x, ms, tokens, q, temp, u, r = _case([4, 2, 3], 9001, "bf16", False, seed)
    want = q4_ref.verify(x, ms, tokens, q, temp, u, r)
    x, tokens, q, temp, u, r = (t.to(cuda) for t in (x, tokens, q, temp, u, r))
    ch = lg.Chunk.of(ms, cuda)
    picked = torch.zeros(sum(ms), dtype=torch.int32, device=cuda)
    accepted = torch.zeros(len(ms), dtype=torch.int32, device=cuda)
    ws = torch.empty(lg.lg_verify_workspace_size(x, ch), dtype=torch.uint8, device=cuda)
    out = torch.full_like(b.qd, 7.0)

    def call(stream):
        lg.lg_chunk_attend(b.cache, b.chunk, 0, b.qd, b.H_q, b.d ** -0.5, 0, 0, out, b.max_len, b.ws, stream)
        lg.lg_verify_draft(x, ch, tokens, q, temp, u, r, picked, accepted, ws, b.cache.status, stream)

    def check():
        assert lg.lg_read_device_status(b.cache) == 0
        assert (picked.tolist(), accepted.tolist()) == want
        ref, tol = b.reference()
        assert ((out.cpu().double() - ref).abs() <= tol).all()
    return call, check


@pytest.mark.parametrize("given", [True, False])
def test_a_stream_of_the_callers_own(cuda, given):
    call, check = _jobs(cuda, 3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    if given:
        call(s)
    else:
        with torch.cuda.stream(s):
            call(None)
    s.synchronize()
    check()


def test_host_threads_at_once(cuda):
    """each thread its own stream and buffers, forty calls without a wait"""
    jobs = [_jobs(cuda, seed) for seed in range(4)]
    torch.cuda.synchronize()
    failed = []

    def work(call):
        try:
            s = torch.cuda.Stream()
            for _ in range(40):
                call(s)
            s.synchronize()
        except Exception as e:
            failed.append(e)
    threads = [threading.Thread(target=work, args=(call,)) for call, _ in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for _, check in jobs:
        check()


@pytest.mark.parametrize("window,sink", [(0, 0), (700, 4)])
def test_a_prompts_chunk_among_single_tokens(cuda, window, sink):
    """one sequence brings 200 rows, one starts with them, the others a token each"""
    rng = np.random.default_rng(2)
    ns = [1500, 200] + [int(n) for n in rng.integers(1, 2500, 14)]
    ms = [200, 200] + [1] * 14
    b = q4_ref.Batch(ns, ms, device=cuda).to_device()
    out = b.attend(window, sink).cpu().double()
    assert lg.lg_read_device_status(b.cache) == 0
    ref, tol = b.reference(window, sink, True)
    assert ((out - ref).abs() <= tol).all()
