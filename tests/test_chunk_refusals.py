"""Addresses that the kernels of include/lg_chunk.h could not use, refused on the host before any
launch."""
import ctypes

import pytest

from paper_2604_10044_gb300 import lg

F = 1 << 20   # a non-null, aligned address that is never dereferenced
by = ctypes.byref


def pick(tokens=F, pmax=F, seen=F, counts=F, allowed=F, off=F, id=F, val=F, status=F, x=F, out=None,
         dtype=1, batch=2, V=100, stride=100):
    lo = lg.LgLogits(x=x, dtype=dtype, batch=batch, V=V, pad=0, stride=stride)
    return lg.lib().lg_pick_token(by(lo), seen, counts, F, by(lg.LgBias(off, id, val)), allowed,
                                  tokens, pmax, out, status, None)


def count(tokens=F, off=F, seen=F, counts=F, status=F, T=4):
    return lg.lib().lg_count_tokens(tokens, off, T, 2, 10, 1, seen, counts, status, None)


@pytest.mark.parametrize("by_bytes", [1, 2, 3])
@pytest.mark.parametrize("name", ["tokens", "pmax", "seen", "counts", "allowed", "off", "id", "val",
                                  "status"])
def test_pick_token_words_off_their_alignment(name, by_bytes):
    assert pick(**{name: F + by_bytes}) == 1


@pytest.mark.parametrize("by_bytes", [1, 2, 3])
@pytest.mark.parametrize("name", ["tokens", "off", "seen", "counts", "status"])
def test_count_tokens_words_off_their_alignment(name, by_bytes):
    assert count(T=0) == 0
    assert count(**{name: F + by_bytes}) == 1


# ------------------------------------------------------------------ outputs over inputs

T, H_Q, H_KV, D = 10, 32, 8, 128
ROW, KV_ROW = H_Q * D * 2, H_KV * D * 2
TOKENS = T * ROW


def cache():
    return lg.LgCache(k=F, v=F, dtype=0, L=2, H_kv=H_KV, d=D, batch=2, S_total=64, seq_off=F, cap=F,
                      len=F, sketch=F, dev_status=F)


def attend(q, out):
    return lg.lib().lg_chunk_attend(by(cache()), by(lg.LgChunk(off=F, T=T, max_new=7)), 0, q, H_Q, 0.1,
                                    0, 0, out, 64, F, 1 << 40, None)


def rope(q, out, k=F << 4, v=F << 5, qs=ROW, ks=KV_ROW, vs=KV_ROW):
    return lg.lib().lg_rope_append(by(cache()), by(lg.LgChunk(off=F, T=T, max_new=7)), 0, q, qs // 2,
                                   H_Q, k, ks // 2, v, vs // 2, F, by(lg.lg_default_rope_params(D)),
                                   out, by(lg.lg_default_params()), None)


@pytest.fixture
def launched():
    """the code of a call that is not refused: of the launch itself, without a GPU"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses of these calls would be dereferenced")
    return 3


def test_attention_over_its_queries(launched):
    q = F << 3
    for out in (q, q + 16, q - 16, q + TOKENS - 16, q - TOKENS + 16):
        assert attend(q, out) == 1
    for out in (q + TOKENS, q - TOKENS):
        assert attend(q, out) == launched


def test_rotated_queries_over_what_is_read(launched):
    q = F << 3
    for out in (q + 16, q - ROW, q + TOKENS - 16, q - TOKENS + 16):
        assert rope(q, out) == 1
    for out in (q, q + TOKENS, q - TOKENS):
        assert rope(q, out) == launched
    # one projection's output, and its first bytes as the result
    packed = ROW + 2 * KV_ROW
    kw = dict(k=q + ROW, v=q + ROW + KV_ROW, qs=packed, ks=packed, vs=packed)
    end = q + T * packed
    for out in (q, q + ROW, end - 16):
        assert rope(q, out, **kw) == 1
    assert rope(q, end, **kw) == launched
    far = F << 6
    for out, ok in ((far, False), (far + T * KV_ROW - 16, False), (far + T * KV_ROW, True)):
        assert rope(q, out, k=far) == (launched if ok else 1)
        assert rope(q, out, v=far) == (launched if ok else 1)


def test_kept_logits_over_the_logits(launched):
    x, kw = F << 3, dict(dtype=1, batch=3, V=100)
    for stride, shift, ok in ((100, 0, True), (100, 1, False), (100, -1, False), (100, 299, False),
                              (100, 300, True), (100, -300, True), (100, -299, False),
                              (200, 100, True), (200, -100, True), (200, 99, False), (200, 101, False),
                              (200, 300, True), (200, 500, True), (250, 100, True), (250, 150, True),
                              (250, 151, False), (250, -100, True), (250, -150, True),
                              (250, -151, False)):
        got = pick(x=x, out=x + 4 * shift, stride=stride, **kw)
        assert got == (launched if ok else 1), (stride, shift)
