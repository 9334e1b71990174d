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
