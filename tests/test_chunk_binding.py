"""What the Python binding of include/lg_chunk.h's calls refuses before anything is launched, without
a GPU: a stand-in for the library notes whether a call reached it."""
from types import SimpleNamespace

import pytest
import torch

from paper_2604_10044_gb300 import lg

I32, BF16 = torch.int32, torch.bfloat16
B, T, H_Q, H_KV, D, V = 3, 5, 4, 2, 64, 70
NW = (V + 31) // 32


class Launched(Exception):
    pass


class On:
    """a tensor that says it is on device 1"""

    def __init__(self, t, dev=1):
        self.t, self.dev = t, dev

    def get_device(self):
        return self.dev

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def call(*a):
        raise Launched
    names = ("lg_begin_chunk", "lg_chunk_attend", "lg_rope_append", "lg_pick_token",
             "lg_count_tokens")
    monkeypatch.setattr(lg, "_lib", SimpleNamespace(**{n: call for n in names}))
    monkeypatch.setattr(lg, "_device", lambda: 1)
    monkeypatch.setattr(lg, "_ptr", lambda t: None if t is None else t.data_ptr())


def z(*shape, dtype=I32):
    return torch.zeros(shape, dtype=dtype)


def _take(tensors, over):
    assert set(over) <= set(tensors)
    tensors.update(over)
    return {n: x if x is None or isinstance(x, On) else On(x) for n, x in tensors.items()}


def _cache_and_chunk(t):
    cache = SimpleNamespace(c=lg.LgCache(batch=B), status=t["status"], d=D, H_kv=H_KV,
                            k=z(1, dtype=BF16), batch=B)
    return cache, lg.Chunk(t["off"], T, T)


def begin(**over):
    t = _take(dict(status=z(1), off=z(B + 1)), over)
    lg.lg_begin_chunk(*_cache_and_chunk(t), stream=0)


def rope(**over):
    t = _take(dict(status=z(1), off=z(B + 1), q=z(T, H_Q, D, dtype=BF16), k=z(T, H_KV, D, dtype=BF16),
                   v=z(T, H_KV, D, dtype=BF16), pos=z(T), out=z(T, H_Q, D, dtype=BF16)), over)
    cache, chunk = _cache_and_chunk(t)
    lg.lg_rope_append(cache, chunk, 0, t["q"], t["k"], t["v"], t["pos"], lg.LgRopeParams(), t["out"],
                      lg.LgGuardParams(), 0)


def attend(**over):
    t = _take(dict(status=z(1), off=z(B + 1), q=z(T, H_Q, D, dtype=BF16),
                   out=z(T, H_Q, D, dtype=BF16), ws=z(1024, dtype=torch.uint8)), over)
    cache, chunk = _cache_and_chunk(t)
    lg.lg_chunk_attend(cache, chunk, 0, t["q"], H_Q, 1.0, 0, 0, t["out"], 8, t["ws"], 0)


def pick(**over):
    f32 = torch.float32
    t = _take(dict(logits=z(B, V, dtype=BF16), seen=z(B, NW), counts=z(B, V),
                   penalty=z(B, 4, dtype=f32), off=z(B + 1), id=z(9), val=z(9, dtype=f32),
                   allowed=z(B, NW), tokens=z(B), pmax=z(B, dtype=f32), status=z(1),
                   kept=z(B, V, dtype=BF16)), over)
    lg.lg_pick_token(t["logits"], t["seen"], t["counts"], t["penalty"], (t["off"], t["id"], t["val"]),
                     t["allowed"], t["tokens"], t["pmax"], t["status"], t["kept"], 0)


def count(**over):
    t = _take(dict(tokens=z(20), off=z(B + 1), seen=z(B, NW), counts=z(B, V), status=z(1)), over)
    lg.lg_count_tokens(t["tokens"], t["off"], V, 1, t["seen"], t["counts"], t["status"], 0)


CALLS = (begin, rope, attend, pick, count)


@pytest.mark.parametrize("call", CALLS)
def test_what_the_header_asks_for_is_passed_on(call):
    with pytest.raises(Launched):
        call()


def test_rows_that_stand_apart_are_passed_on():
    qkv = z(T, H_Q + 2 * H_KV, D, dtype=BF16)
    with pytest.raises(Launched):
        rope(q=qkv[:, :H_Q], k=qkv[:, H_Q:H_Q + H_KV], v=qkv[:, H_Q + H_KV:])
    wide = z(B, V + 6, dtype=BF16)
    with pytest.raises(Launched):
        pick(logits=wide[:, 2:V + 2], kept=z(B, V + 6, dtype=BF16)[:, :V])


@pytest.mark.parametrize("name,heads", [("q", H_Q), ("k", H_KV), ("v", H_KV)])
def test_tokens_whose_rows_overlap(name, heads):
    """one row for all tokens, and rows that begin within the one before"""
    for bad in (z(1, heads, D, dtype=BF16).expand(T, heads, D),
                z(heads * D * 4, dtype=BF16).as_strided((T, heads, D), (D // 2, D, 1))):
        with pytest.raises(ValueError):
            rope(**{name: bad})


def test_logits_whose_rows_overlap():
    for bad in (z(1, V, dtype=BF16).expand(B, V), z(4 * V, dtype=BF16).as_strided((B, V), (V // 2, 1))):
        with pytest.raises(ValueError):
            pick(logits=bad, kept=None)
        with pytest.raises(ValueError):
            pick(logits=bad, kept=bad)


def test_one_row_may_have_any_stride():
    """the stride between rows says nothing of one"""
    assert lg._rows_stride(z(H_Q * D).as_strided((1, H_Q, D), (1, D, 1)), "q") == H_Q * D
    assert lg._rows_stride(z(H_Q * D + 9).as_strided((1, H_Q, D), (H_Q * D + 9, D, 1)), "q") == H_Q * D


def _sliced(t):
    """the same shape and values, every second element of a larger tensor"""
    return torch.stack([t, t], -1)[..., 0]


def _broadcast(t):
    """the same shape from one element"""
    return t.reshape(-1)[:1].expand(t.numel()).view(t.shape) if t.dim() == 1 else \
        t[:1].expand(t.shape)


DENSE = {begin: ["off"], rope: ["off", "pos", "out"], attend: ["off", "q", "out"],
         pick: ["seen", "counts", "penalty", "off", "id", "val", "allowed", "tokens", "pmax"],
         count: ["tokens", "off", "seen", "counts"]}


@pytest.mark.parametrize("call,name", [(c, n) for c in CALLS for n in DENSE[c]])
def test_tensors_that_are_not_dense(call, name):
    """a slice of a larger tensor; one element or row for all of them"""
    shapes = dict(seen=z(B, NW), counts=z(B, V), allowed=z(B, NW), penalty=z(B, 4, dtype=torch.float32),
                  id=z(9), val=z(9, dtype=torch.float32), pmax=z(B, dtype=torch.float32),
                  pos=z(T), out=z(T, H_Q, D, dtype=BF16), q=z(T, H_Q, D, dtype=BF16), off=z(B + 1),
                  tokens=z(20) if call is count else z(B))
    for bad in (_sliced(shapes[name]), _broadcast(shapes[name])):
        assert bad.shape == shapes[name].shape and not bad.is_contiguous()
        with pytest.raises(ValueError):
            call(**{name: bad})


@pytest.mark.parametrize("call,name,bad", [
    (pick, "seen", z(B, NW + 1)), (pick, "counts", z(B, V + 2)), (pick, "allowed", z(B, NW + 1)),
    (pick, "penalty", z(B, 8, dtype=torch.float32)), (count, "seen", z(B, NW + 1)),
    (count, "counts", z(B, V + 2))])
def test_rows_of_another_length(call, name, bad):
    """long enough, but row b does not begin where the kernels take it from"""
    with pytest.raises(ValueError):
        call(**{name: bad})


def test_more_rows_and_flat_rows_are_passed_on():
    with pytest.raises(Launched):
        pick(seen=z(B + 2, NW), counts=z((B + 1) * V), allowed=z(B * NW), tokens=z(B + 4))
    with pytest.raises(Launched):
        count(seen=z(B * NW), counts=z(B + 2, V))


def test_workspaces_and_status_words():
    with pytest.raises(ValueError):
        attend(ws=z(2048, dtype=torch.uint8)[::2])
    for call in (pick, count):
        for bad in (z(0), z(1, dtype=torch.int64)):
            with pytest.raises(ValueError):
                call(status=bad)
        with pytest.raises(Launched):
            call(status=None)


@pytest.mark.parametrize("name,bad", [
    ("k", z(T - 1, H_KV * 2, D, dtype=BF16)), ("k", z(1, T * H_KV, D, dtype=BF16)),
    ("k", z(T, H_KV * 2, D // 2, dtype=BF16)), ("k", z(2 * T, H_KV - 1, D, dtype=BF16)),
    ("v", z(T - 1, H_KV, D * 2, dtype=BF16)), ("v", z(T * 2, H_KV, D // 2, dtype=BF16)),
    ("q", z(T - 1, H_Q, D * 2, dtype=BF16)), ("q", z(T, H_Q, D * 2, dtype=BF16)),
    ("q", z(T * 2, H_Q, D // 2, dtype=BF16))])
def test_tokens_of_another_shape(name, bad):
    """as many elements as are needed, but in fewer rows, or of heads of another size or number"""
    with pytest.raises(ValueError):
        rope(**{name: bad}, **(dict(out=z(4 * T, H_Q, D, dtype=BF16)) if name == "q" else {}))


@pytest.mark.parametrize("call", [begin, rope, attend])
def test_offsets_of_fewer_sequences(call):
    with pytest.raises(ValueError):
        call(off=z(B))
    with pytest.raises(Launched):
        call(off=z(B + 3))


ALL = {begin: ["status", "off"], rope: ["off", "q", "k", "v", "pos", "out"],
       attend: ["off", "q", "out", "ws"],
       pick: ["logits", "seen", "counts", "penalty", "off", "id", "val", "allowed", "tokens", "pmax",
              "status", "kept"],
       count: ["tokens", "off", "seen", "counts", "status"]}


@pytest.mark.parametrize("call,name", [(c, n) for c in CALLS for n in ALL[c]])
@pytest.mark.parametrize("dev", [-1, 0, 2])
def test_one_tensor_on_another_device(call, name, dev):
    """any of them, on the CPU or on another GPU than the current one"""
    shapes = dict(q=z(T, H_Q, D, dtype=BF16), k=z(T, H_KV, D, dtype=BF16), v=z(T, H_KV, D, dtype=BF16),
                  out=z(T, H_Q, D, dtype=BF16), ws=z(1024, dtype=torch.uint8), pos=z(T), off=z(B + 1),
                  logits=z(B, V, dtype=BF16), kept=z(B, V, dtype=BF16), seen=z(B, NW), counts=z(B, V),
                  allowed=z(B, NW), penalty=z(B, 4, dtype=torch.float32), id=z(9),
                  val=z(9, dtype=torch.float32), pmax=z(B, dtype=torch.float32), status=z(1),
                  tokens=z(20) if call is count else z(B))
    with pytest.raises(ValueError):
        call(**{name: On(shapes[name], dev)})
