"""include/lg_chunk.h without a GPU: declarations, exports and ctypes signatures agree; defaults;
every refusal happens on the host before any launch, with the documented code."""
import ctypes
import inspect
import os
import re
from types import SimpleNamespace

import pytest
import torch

from paper_2604_10044_gb300 import lg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = 1 << 20   # a non-null, aligned address that is never dereferenced
by = ctypes.byref


def declarations():
    src = open(os.path.join(ROOT, "include", "lg_chunk.h")).read()
    src = re.sub(r"/\*.*?\*/", " ", src, flags=re.S)
    return {m.group(1): m.group(2) for m in
            re.finditer(r"^LG_API [^(]*?\b(lg_\w+)\(([^)]*)\)\s*;", src, flags=re.M)}


def test_declarations_exports_and_wrappers_agree():
    decl = declarations()
    assert sorted(decl) == sorted(lg.chunk_symbols())
    L = lg.lib()
    for name, params in decl.items():
        assert len(getattr(L, name).argtypes) == params.count(",") + 1, name
        wrapper = inspect.signature(getattr(lg, name)).parameters
        if "cudaStream_t" in params:
            last = list(wrapper.values())[-1]
            assert last.name == "stream" and last.default is None, name


def test_struct_sizes():
    """as the C compiler lays them out (fields are naturally aligned in the order of the header)"""
    assert ctypes.sizeof(lg.LgChunk) == 16
    assert ctypes.sizeof(lg.LgRopeParams) == 16 + 7 * 8
    assert ctypes.sizeof(lg.LgLogits) == 32
    assert ctypes.sizeof(lg.LgBias) == 24


def test_defaults():
    p = lg.lg_default_rope_params(128)
    assert (p.layout, p.rot, p.scaling, p.orig_len) == (lg.LG_ROPE_HALF, 128, lg.LG_ROPE_PLAIN, 8192)
    assert (p.theta, p.factor, p.low, p.high, p.beta_fast, p.beta_slow, p.mscale) == (
        10000.0, 1.0, 1.0, 4.0, 32.0, 1.0, 1.0)
    assert lg.lib().lg_default_rope_params(None, 128) == 1
    assert lg.lib().lg_default_rope_params(by(p), 8) == 1


def _cache(**over):
    c = lg.LgCache(k=F, v=F, dtype=0, L=2, H_kv=8, d=128, batch=2, S_total=64, seq_off=F, cap=F,
                   len=F, sketch=F, dev_status=F)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def _chunk(**over):
    ch = lg.LgChunk(off=F, T=10, max_new=7)
    for k, v in over.items():
        setattr(ch, k, v)
    return ch


def test_begin_chunk_refusals():
    f = lg.lib().lg_begin_chunk
    c, ch = _cache(), _chunk()
    assert f(None, by(ch), None) == 1
    assert f(by(c), None, None) == 1
    assert f(by(_cache(d=96)), by(ch), None) == 2
    for bad in (dict(off=None), dict(off=F + 2), dict(T=-1), dict(max_new=-1)):
        assert f(by(c), by(_chunk(**bad)), None) == 1, bad


def _rope(cache=None, chunk=None, layer=0, q=F, qs=4096, H_q=32, k=F, ks=1024, v=F, vs=1024, pos=F,
          out=F + 4096, params=None, **rope):
    rp = lg.lg_default_rope_params(128, **rope)
    return lg.lib().lg_rope_append(by(cache or _cache()), by(chunk or _chunk()), layer, q, qs, H_q,
                                   k, ks, v, vs, pos, by(rp), out,
                                   by(params or lg.lg_default_params()), None)


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), 1), (dict(layer=-1), 1), (dict(H_q=-1), 1), (dict(q=None), 1),
    (dict(out=None), 1), (dict(H_q=0), 1), (dict(k=None), 1), (dict(v=None), 1),
    (dict(pos=None), 1), (dict(q=F + 8), 1), (dict(k=F + 2), 1), (dict(v=F + 4), 1),
    (dict(out=F + 8), 1), (dict(pos=F + 2), 1), (dict(qs=4095), 1), (dict(qs=4104 + 4), 1),
    (dict(ks=1016), 1), (dict(ks=1028), 1), (dict(vs=512), 1), (dict(out=F, qs=8192), 1),
    (dict(rot=0), 2), (dict(rot=130), 2), (dict(rot=144), 2), (dict(rot=24), 2), (dict(rot=-16), 2),
    (dict(layout=2), 1), (dict(scaling=5), 1), (dict(scaling=-1), 1), (dict(theta=1.0), 1),
    (dict(theta=float("nan")), 1), (dict(theta=float("inf")), 1), (dict(mscale=0.0), 1),
    (dict(mscale=float("inf")), 1), (dict(scaling=1, factor=0.5), 1),
    (dict(scaling=2, factor=float("nan")), 1), (dict(scaling=3, low=4.0), 1),
    (dict(scaling=3, low=0.0), 1), (dict(scaling=3, orig_len=0), 1),
    (dict(scaling=4, beta_slow=0.0), 1), (dict(scaling=4, beta_fast=1.0), 1),
    (dict(scaling=4, orig_len=0), 1)])
def test_rope_append_refusals(kw, code):
    assert _rope(**kw) == code


def test_rope_append_of_no_rows_launches_nothing():
    assert _rope(chunk=_chunk(T=0)) == 0


def _attend(cache=None, chunk=None, layer=0, q=F, H_q=32, scale=0.1, window=0, sink=0,
            out=F + 65536, max_len=64, ws=F, ws_bytes=1 << 40):
    return lg.lib().lg_chunk_attend(by(cache or _cache()), by(chunk or _chunk()), layer, q, H_q,
                                    scale, window, sink, out, max_len, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), 1), (dict(H_q=30), 1), (dict(H_q=0), 1), (dict(H_q=72), 2),
    (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(window=-1), 1), (dict(sink=-1), 1), (dict(max_len=0), 1), (dict(q=None), 1),
    (dict(out=None), 1), (dict(q=F + 8), 1), (dict(out=F + 8), 1), (dict(out=F), 1),
    (dict(ws=None), 6), (dict(ws=F + 16), 6), (dict(ws_bytes=1), 6),
    (dict(cache=_cache(S_total=1 << 28)), 2), (dict(cache=_cache(dtype=3)), 2),
    (dict(chunk=_chunk(off=None)), 1)])
def test_chunk_attend_refusals(kw, code):
    assert _attend(**kw) == code


def test_chunk_attend_of_no_rows_launches_nothing():
    assert _attend(chunk=_chunk(T=0)) == 0 and _attend(chunk=_chunk(max_new=0)) == 0


def test_workspace_size():
    f = lg.lib().lg_chunk_workspace_size
    assert f(by(_cache()), by(_chunk()), 30, 64) == 0
    assert f(by(_cache()), by(_chunk()), 32, 0) == 0
    n = f(by(_cache()), by(_chunk()), 32, 64)
    assert n > 0 and n % 256 == 0
    assert _attend(ws_bytes=n - 1) == 6


def _pick(x=F, dtype=1, batch=2, V=100, stride=100, seen=F, counts=F, pen=F, bias=None, allowed=F,
          tokens=F, pmax=F, out=None):
    lo = lg.LgLogits(x=x, dtype=dtype, batch=batch, V=V, pad=0, stride=stride)
    return lg.lib().lg_pick_token(by(lo), seen, counts, pen, bias, allowed, tokens, pmax, out, None,
                                  None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), 1), (dict(tokens=None), 1), (dict(pmax=None), 1), (dict(dtype=2), 2),
    (dict(batch=0), 1), (dict(V=0), 1), (dict(stride=99), 1), (dict(V=1 << 21, stride=1 << 21), 2),
    (dict(x=F + 2), 1), (dict(out=F + 2), 1), (dict(counts=None), 1), (dict(seen=None), 1),
    (dict(pen=None), 1), (dict(pen=F + 4), 1), (dict(bias=lg.LgBias(off=F, id=F, val=None)), 1),
    (dict(bias=lg.LgBias(off=None, id=F, val=F)), 1)])
def test_pick_token_refusals(kw, code):
    assert _pick(**kw) == code


def test_count_tokens_refusals():
    f = lg.lib().lg_count_tokens
    assert f(None, F, 4, 2, 10, 1, F, F, None, None) == 1
    assert f(F, F, 4, 2, 10, 1, None, F, None, None) == 1
    assert f(F, F, 4, 2, 10, 1, F, None, None, None) == 1
    assert f(F, F, -1, 2, 10, 1, F, F, None, None) == 1
    assert f(F, None, 4, 2, 10, 1, F, F, None, None) == 1   # one token a row: T is the batch
    assert f(F, F, 4, 0, 10, 1, F, F, None, None) == 1
    assert f(F, F, 4, 2, 0, 1, F, F, None, None) == 1
    assert f(F, F, 0, 2, 10, 1, F, F, None, None) == 0


def test_binding_refuses_tensors_that_the_kernels_cannot_read(monkeypatch):
    """another device than the current one, another type than the cache's, too few elements"""
    z, i32 = torch.zeros, torch.int32

    class At:  # a tensor on a device of one's choice
        def __init__(self, t, dev):
            self.t, self.dev, self.device = t, dev, "cuda:%d" % dev

        def get_device(self):
            return self.dev

        def __getattr__(self, name):
            return getattr(self.t, name)

    def args(dev=1, **over):
        t = dict(status=z(1, dtype=i32), off=z(2, dtype=i32), q=z(3, 4, 64), k=z(3, 2, 64),
                 v=z(3, 2, 64), pos=z(3, dtype=i32), out=z(3, 4, 64), ws=z(64))
        t = {n: At(x, dev) for n, x in t.items()}
        t.update(over)
        cache = SimpleNamespace(c=lg.LgCache(), status=t["status"], d=64, H_kv=2, k=z(1))
        chunk = SimpleNamespace(c=lg.LgChunk(), off=t["off"], T=3, max_new=3)
        return cache, chunk, t

    def attend(*a, **over):
        cache, chunk, t = args(*a, **over)
        lg.lg_chunk_attend(cache, chunk, 0, t["q"], 4, 1.0, 0, 0, t["out"], 8, t["ws"], 0)

    def rope(*a, **over):
        cache, chunk, t = args(*a, **over)
        lg.lg_rope_append(cache, chunk, 0, t["q"], t["k"], t["v"], t["pos"], lg.LgRopeParams(),
                          t["out"], lg.LgGuardParams(), 0)

    def pick(dev=1, **over):
        t = dict(logits=z(2, 33), seen=z(4, dtype=i32), counts=z(66, dtype=i32), penalty=z(2, 4),
                 allowed=z(4, dtype=i32), tokens=z(2, dtype=i32), pmax=z(2))
        t = {n: At(x, dev) for n, x in t.items()}
        t.update(over)
        lg.lg_pick_token(t["logits"], t["seen"], t["counts"], t["penalty"], None, t["allowed"],
                         t["tokens"], t["pmax"], stream=0)

    def count(dev=1, **over):
        t = dict(tokens=z(2, dtype=i32), seen=z(4, dtype=i32), counts=z(66, dtype=i32))
        t = {n: At(x, dev) for n, x in t.items()}
        t.update(over)
        lg.lg_count_tokens(t["tokens"], None, 33, 1, t["seen"], t["counts"], stream=0)

    class Launched(Exception):
        pass

    def call(*a):
        raise Launched

    names = ("lg_chunk_attend", "lg_rope_append", "lg_pick_token", "lg_count_tokens")
    monkeypatch.setattr(lg, "_lib", SimpleNamespace(**{n: call for n in names}))
    monkeypatch.setattr(lg, "_device", lambda: 1)
    for f in (attend, rope, pick, count):
        with pytest.raises(Launched):
            f()
        for dev in (-1, 0, 2):
            with pytest.raises(ValueError):
                f(dev)
    bad = {attend: dict(q=[z(3, 4, 64, dtype=torch.bfloat16), z(2, 4, 64)], out=[z(3, 2, 64)]),
           rope: dict(q=[z(2, 4, 64)], k=[z(3, 2, 32), z(3, 2, 64).double()], v=[z(1, 2, 64)],
                      pos=[z(2, dtype=i32), z(3)], out=[z(3, 3, 64), z(3, 4, 64).double()]),
           pick: dict(seen=[z(3, dtype=i32)], counts=[z(65, dtype=i32), z(66)], penalty=[z(7)],
                      allowed=[z(3, dtype=i32), z(4).double()],
                      tokens=[z(1, dtype=i32), z(2)], pmax=[z(1), z(2, dtype=torch.bfloat16)]),
           count: dict(tokens=[z(2)], seen=[z(3, dtype=i32)], counts=[z(65, dtype=i32)])}
    for f, cases in bad.items():
        for name, values in cases.items():
            for v in values:
                with pytest.raises(ValueError):
                    f(**{name: At(v, 1)})


def test_binding_refuses_broken_rows():
    x = torch.zeros(3, 4, 8)
    assert lg._rows_stride(x, "x") == 32
    assert lg._rows_stride(torch.zeros(3, 10, 8)[:, 2:6], "x") == 80
    assert lg._rows_stride(torch.zeros(1, 10, 8)[:, 2:6], "x") >= 32
    for bad in (x.transpose(0, 1), torch.zeros(3, 4, 16)[..., ::2], torch.zeros(3, 4, 16)[..., :8],
                torch.zeros(3, 32)):
        with pytest.raises(ValueError):
            lg._rows_stride(bad, "x")
    with pytest.raises(ValueError):
        lg.lg_chunk_attend(None, None, 0, x.transpose(0, 1), 4, 1.0, 0, 0, x, 8, x)
    with pytest.raises(ValueError):
        lg.lg_rope_append(None, None, 0, x, x, x, x, None, x.transpose(0, 1), None)
    with pytest.raises(ValueError):
        lg.lg_pick_token(torch.zeros(3, 8).t(), None, None, None, None, None, None, None)
    with pytest.raises(ValueError):
        lg.lg_pick_token(torch.zeros(3, 8), None, None, None, None, None, None, None,
                         logits_out=torch.zeros(3, 9)[:, :8])
