"""include/lg_draft.h without a GPU: declarations, exports and wrappers agree, and what the calls refuse
on the host before any launch; the same for a 4-bit cache through the calls of lg.h and lg_chunk.h."""
import ctypes
import inspect
import os
import re

import pytest
import torch

from paper_2604_10044_gb300 import lg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = 1 << 20   # a non-null, aligned address that is never dereferenced
by = ctypes.byref


def declarations():
    src = open(os.path.join(ROOT, "include", "lg_draft.h")).read()
    src = re.sub(r"/\*.*?\*/", " ", src, flags=re.S)
    return {m.group(1): m.group(2) for m in
            re.finditer(r"^LG_API [^(]*?\b(lg_\w+)\(([^)]*)\)\s*;", src, flags=re.M)}


def test_declarations_exports_and_wrappers_agree():
    decl = declarations()
    assert sorted(decl) == sorted(lg.draft_symbols())
    L = lg.lib()
    for name, params in decl.items():
        assert len(getattr(L, name).argtypes) == params.count(",") + 1, name
        if "cudaStream_t" in params:
            last = list(inspect.signature(getattr(lg, name)).parameters.values())[-1]
            assert last.name == "stream" and last.default is None, name


T, B, V = 10, 3, 100


def rows(x=F, dtype=1, batch=T, V=V, stride=V):
    return lg.LgLogits(x=x, dtype=dtype, batch=batch, V=V, pad=0, stride=stride)


def verify(x=None, draft=None, ch=None, batch=B, tokens=F << 4, temp=None, u=F << 4, r=F << 4,
           picked=F << 5, accepted=F << 6, ws=F << 7, n=1 << 30, status=None):
    x = rows() if x is None else x
    ch = lg.LgChunk(off=F << 4, T=T, max_new=5) if ch is None else ch
    p = lambda a: None if a is None or a == 0 else ctypes.addressof(a)
    return lg.lib().lg_verify_draft(p(x), None if ch == 0 else by(ch), batch, tokens, p(draft), temp, u,
                                    r, picked, accepted, ws, n, status, None)


def test_verify_refusals():
    small = rows(batch=T - 1)
    for kw, code in [
            (dict(x=0), 1), (dict(x=rows(x=None)), 1), (dict(x=rows(dtype=2)), 2),
            (dict(x=rows(V=0)), 1), (dict(x=rows(stride=V - 1)), 1), (dict(x=small), 1),
            (dict(x=rows(V=(1 << 20) + 1, stride=1 << 21)), 2), (dict(x=rows(x=F + 2)), 1),
            (dict(draft=small), 1), (dict(draft=rows(V=V - 1)), 1), (dict(draft=rows(dtype=7)), 2),
            (dict(draft=rows(x=F + 1, dtype=0)), 1), (dict(ch=0), 1),
            (dict(ch=lg.LgChunk(off=None, T=T, max_new=5)), 1),
            (dict(ch=lg.LgChunk(off=F, T=-1, max_new=5)), 1),
            (dict(ch=lg.LgChunk(off=F, T=T, max_new=-1)), 1),
            (dict(ch=lg.LgChunk(off=F, T=65536, max_new=5), x=rows(batch=65536)), 2),
            (dict(batch=0), 1), (dict(tokens=None), 1), (dict(u=None), 1), (dict(r=None), 1),
            (dict(picked=None), 1), (dict(accepted=None), 1), (dict(tokens=F + 2), 1),
            (dict(u=F + 1), 1), (dict(r=F + 3), 1), (dict(temp=F + 2), 1), (dict(picked=F + 1), 1),
            (dict(accepted=F + 2), 1), (dict(status=F + 1), 1), (dict(ws=None), 6), (dict(n=8), 6),
            (dict(ws=F + 8), 6),
            # results over what is read, or over one another
            (dict(picked=F), 1), (dict(accepted=F + 4 * (T * V - 1)), 1), (dict(picked=(F << 4) + 36), 1),
            (dict(accepted=(F << 5) + 4 * T - 4), 1), (dict(temp=(F << 6) + 4), 1),
            (dict(draft=rows(x=F << 5)), 1), (dict(picked=F << 7), 1)]:
        assert verify(**kw) == code, kw
    assert verify(ch=lg.LgChunk(off=F, T=0, max_new=0), ws=None) == 6
    L = lg.lib()
    assert L.lg_verify_workspace_size(None, by(lg.LgChunk(off=F, T=T, max_new=5))) == 0
    assert L.lg_verify_workspace_size(ctypes.addressof(rows()), None) == 0


def cache(**over):
    f = dict(k=F, v=F, dtype=lg.LG_Q4, L=2, H_kv=8, d=128, batch=2, S_total=64, seq_off=F, cap=F, len=F,
             sketch=F, dev_status=F)
    f.update(over)
    return lg.LgCache(**f)


def test_calls_that_a_4_bit_cache_refuses():
    L, p = lg.lib(), by(lg.lg_default_params())
    assert L.lg_begin_step(by(cache(h2o=F, pos=F)), None) == 2
    assert L.lg_sketch_build(by(cache()), p, 10, None) == 2
    assert L.lg_h2o_reset(by(cache()), 10, None) == 1
    assert L.lg_h2o_evict(by(cache()), F, F, 10, None) == 1
    assert L.lg_streaming_evict(by(cache()), F, F, 4, 10, None) == 1
    attend = lambda h2o=0, n=1 << 30, H_q=32: L.lg_decode_attend(
        by(cache()), 0, 1, F, H_q, 0.1, F, F, 64, h2o, 100, F, n, None)
    assert attend(h2o=1) == 1 and attend(n=16) == 6 and attend(H_q=9) == 1 and attend(H_q=72) == 2
    assert L.lg_workspace_size(by(cache()), 32, 1, 100, 1) == 0
    assert L.lg_workspace_size(by(cache()), 9, 1, 100, 0) == 0
    assert L.lg_workspace_size(by(cache()), 32, 1, 100, 0) % 256 == 0
    with pytest.raises(ValueError):
        lg.Cache(1, 2, 64, "q4", [0], [4], [0], "cpu", "h2o")


def test_read_rows_and_end_chunk_refusals():
    L, ch = lg.lib(), lg.LgChunk(off=F, T=T, max_new=5)
    read = lambda c=None, ch=ch, layer=0, k=F << 4, v=F << 6: L.lg_read_rows(
        by(c or cache()), by(ch), layer, k, v, None)
    assert read(c=cache(dtype=0)) == 2 and read(layer=2) == 1 and read(layer=-1) == 1
    assert read(k=None) == 1 and read(v=None) == 1 and read(k=F + 8) == 1
    assert read(v=(F << 4) + 16) == 1 and read(ch=lg.LgChunk(off=F, T=0, max_new=5)) == 0
    assert L.lg_end_chunk(by(cache()), by(ch), None, None) == 1
    assert L.lg_end_chunk(by(cache()), by(ch), F + 2, None) == 1
    assert L.lg_end_chunk(by(cache()), None, F, None) == 1


def test_chunk_attend_over_four_bits_wants_its_workspace():
    L = lg.lib()
    for new in (1, 5, 16, 17, 512):
        ch = lg.LgChunk(off=F, T=600, max_new=new)
        n = L.lg_chunk_workspace_size(by(cache()), by(ch), 32, 64)
        assert n > 0 and n % 256 == 0
        assert L.lg_chunk_attend(by(cache()), by(ch), 0, F << 6, 32, 0.1, 0, 0, F << 8, 64, F, n - 256,
                                 None) == 6
        for window in (1, 100):
            assert L.lg_chunk_attend(by(cache()), by(ch), 0, F << 6, 32, 0.1, window, 0, F << 8, 64, F,
                                     n - 256, None) == 6
    assert L.lg_chunk_attend(by(cache()), by(ch), 0, F << 6, 32, 0.1, 0, 0, (F << 6) + 16, 64, F, 1 << 40,
                             None) == 1


# ------------------------------------------------------------------ the binding

def test_the_binding_refuses_what_is_not_dense_or_elsewhere(monkeypatch):
    at = [-1]  # the "current device" is the CPU
    monkeypatch.setattr(lg, "_device", lambda: at[0])
    called = []
    class Lib:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0
    monkeypatch.setattr(lg, "_lib", Lib())
    monkeypatch.setattr(lg, "_raw_stream", None)
    monkeypatch.setattr(lg, "_stream", lambda s: 0)
    z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype)
    f = lambda *s: z(*s, dtype=torch.float32)
    ch = lg.Chunk(z(B + 1), T, 5)

    def call(**over):
        t = dict(logits=f(T, V), tokens=z(T), draft=f(T, V), temp=f(B), u=f(T), r=f(B), picked=z(T),
                 accepted=z(B), ws=z(999, dtype=torch.uint8), status=z(1))
        t.update(over)
        lg.lg_verify_draft(t["logits"], ch, t["tokens"], t["draft"], t["temp"], t["u"], t["r"],
                           t["picked"], t["accepted"], t["ws"], t["status"])

    call()
    call(draft=None, temp=None, status=None)
    call(logits=f(T, V + 5)[:, 2:V + 2])
    n = len(called)
    for name, bad in [("logits", f(1, V).expand(T, V)), ("logits", f(V, T).T), ("logits", f(T * V)),
                      ("draft", f(1, V).expand(T, V)), ("tokens", z(T - 1)), ("tokens", f(T)),
                      ("tokens", z(2 * T)[::2]), ("temp", f(B - 1)), ("u", f(T - 1)), ("u", z(T)),
                      ("r", f(2 * B)[::2]), ("picked", z(T - 1)), ("accepted", z(B - 1)),
                      ("ws", z(64, 2)[:, 0]), ("status", f(1))]:
        with pytest.raises(ValueError):
            call(**{name: bad})
    at[0] = 0  # another device than the tensors'
    with pytest.raises(ValueError):
        call()
    assert len(called) == n
