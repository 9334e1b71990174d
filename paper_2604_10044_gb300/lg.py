"""Python binding of liblg.so (include/lg.h, lg_chunk.h, lg_draft.h): argument marshalling only.

Every function named ``lg_*`` here calls the C function of the same name with raw device
pointers taken from torch tensors and the caller's CUDA stream; every step of the decode path
runs in the library's kernels.  ``Cache`` and ``Guard`` bundle the device buffers of one batch
and issue a whole guarded decode step in the order the ABI documents.  There is no CPU path:
loading fails loudly when the shared library is missing.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblg.so")

LG_OK, LG_BF16, LG_F32, LG_Q4 = 0, 0, 1, 2
STATUS = {0: "LG_OK", 1: "LG_ERR_INVALID_ARG", 2: "LG_ERR_UNSUPPORTED", 3: "LG_ERR_CUDA",
          4: "LG_ERR_CAPACITY", 5: "LG_ERR_TIMEOUT", 6: "LG_ERR_WORKSPACE", 7: "LG_ERR_BUDGET"}


class LgError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__("%s -> %s" % (fn, STATUS.get(code, code)))
        self.code = code


class LgCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("L", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("pad", ctypes.c_int32), ("S_total", ctypes.c_int64),
                ("seq_off", ctypes.c_void_p), ("cap", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("sketch", ctypes.c_void_p), ("h2o", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("dev_status", ctypes.c_void_p)]


class LgGuardParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "W", "K", "t_min", "cooldown", "n_anchor", "stall_len", "p_min", "p_max", "l_min",
        "m_rep", "suffix_w", "guard_layer", "level_max", "retrig_window", "headroom", "pad")] + \
        [(n, ctypes.c_double) for n in ("theta_ttr", "theta_nov", "theta_ent", "theta_lift",
                                         "tau_ham")]


class LgTokenParams(ctypes.Structure):
    _fields_ = [("cr_every", ctypes.c_int32), ("theta_streak", ctypes.c_int32),
                ("hist", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("theta_cr", ctypes.c_double), ("theta_conf", ctypes.c_double)]


class LgChunk(ctypes.Structure):
    _fields_ = [("off", ctypes.c_void_p), ("T", ctypes.c_int32), ("max_new", ctypes.c_int32)]


class LgRopeParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("layout", "rot", "scaling", "orig_len")] + \
        [(n, ctypes.c_double) for n in ("theta", "factor", "low", "high", "beta_fast",
                                         "beta_slow", "mscale")]


class LgLogits(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("V", ctypes.c_int32), ("pad", ctypes.c_int32), ("stride", ctypes.c_int64)]


class LgBias(ctypes.Structure):
    _fields_ = [("off", ctypes.c_void_p), ("id", ctypes.c_void_p), ("val", ctypes.c_void_p)]


LG_ROPE_HALF, LG_ROPE_INTERLEAVED = 0, 1
LG_ROPE_PLAIN, LG_ROPE_LINEAR, LG_ROPE_BASE, LG_ROPE_BANDS, LG_ROPE_YARN = range(5)

STATE_BYTES = 32  # lg_guard_state: 8 x int32
STATE_WORD_N_INT = 4  # lg_guard_state.n_int: interventions so far

_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("liblg.so is not built (run __graft_entry__.build()); "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, P = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.POINTER
        sig = {
            "lg_default_params": [P(LgGuardParams)],
            "lg_workspace_size": [P(LgCache), i32, i32, i32, i32],
            "lg_state_init": [P(LgCache), vp, i32, vp],
            "lg_begin_step": [P(LgCache), vp],
            "lg_append": [P(LgCache), i32, i32, vp, vp, vp, P(LgGuardParams), vp],
            "lg_sketch_build": [P(LgCache), P(LgGuardParams), i32, vp],
            "lg_decode_attend": [P(LgCache), i32, i32, vp, i32, ctypes.c_float, vp, vp, i32, i32,
                                 i32, vp, ctypes.c_size_t, vp],
            "lg_detect": [P(LgCache), vp, i32, vp, vp, P(LgGuardParams), vp, vp, vp, vp, vp],
            "lg_detect_state_size": [P(LgCache), P(LgGuardParams)],
            "lg_detect_prune": [P(LgCache), vp, i32, vp, vp, P(LgGuardParams), vp, vp, vp, vp,
                                vp, vp, i32, i32, vp],
            "lg_default_token_params": [P(LgTokenParams)],
            "lg_token_state_size": [P(LgCache), P(LgGuardParams), P(LgTokenParams)],
            "lg_token_detect": [P(LgCache), vp, vp, vp, vp, i32, vp, P(LgGuardParams),
                                P(LgTokenParams), vp, vp, vp, vp, vp],
            "lg_token_detect_prune": [P(LgCache), vp, vp, vp, vp, P(LgGuardParams),
                                      P(LgTokenParams), vp, vp, vp, vp, vp, vp, i32, i32, vp],
            "lg_prune_compact": [P(LgCache), vp, vp, vp, vp, P(LgGuardParams), vp, vp, i32, i32,
                                 vp],
            "lg_h2o_reset": [P(LgCache), i32, vp],
            "lg_h2o_evict": [P(LgCache), vp, vp, i32, vp],
            "lg_streaming_evict": [P(LgCache), vp, vp, i32, i32, vp],
            "lg_read_device_status": [P(LgCache), vp, vp],
            "lg_decode_attend_noalloc": [P(LgCache), i32, i32, vp, i32, ctypes.c_float, vp, vp,
                                         i32, i32, i32, vp],
            "lg_status_string": [i32],
            "lg_begin_chunk": [P(LgCache), P(LgChunk), vp],
            "lg_default_rope_params": [P(LgRopeParams), i32],
            "lg_rope_append": [P(LgCache), P(LgChunk), i32, vp, i64, i32, vp, i64, vp, i64, vp,
                               P(LgRopeParams), vp, P(LgGuardParams), vp],
            "lg_chunk_workspace_size": [P(LgCache), P(LgChunk), i32, i32],
            "lg_chunk_attend": [P(LgCache), P(LgChunk), i32, vp, i32, ctypes.c_float, i32, i32, vp,
                                i32, vp, ctypes.c_size_t, vp],
            "lg_count_tokens": [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp],
            "lg_pick_token": [vp, vp, vp, vp, P(LgBias), vp, vp, vp, vp, vp, vp],
            "lg_verify_workspace_size": [vp, P(LgChunk)],
            "lg_verify_draft": [vp, P(LgChunk), i32, vp, vp, vp, vp, vp, vp, vp, vp,
                                ctypes.c_size_t, vp, vp],
            "lg_end_chunk": [P(LgCache), P(LgChunk), vp, vp],
            "lg_read_rows": [P(LgCache), P(LgChunk), i32, vp, vp, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        L.lg_workspace_size.restype = ctypes.c_size_t
        L.lg_detect_state_size.restype = ctypes.c_size_t
        L.lg_chunk_workspace_size.restype = ctypes.c_size_t
        L.lg_token_state_size.restype = ctypes.c_size_t
        L.lg_verify_workspace_size.restype = ctypes.c_size_t
        L.lg_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def exported_symbols():
    """names of the C ABI functions declared in include/lg.h"""
    return ["lg_default_params", "lg_status_string", "lg_workspace_size", "lg_state_init",
            "lg_begin_step", "lg_append", "lg_sketch_build", "lg_decode_attend", "lg_detect",
            "lg_prune_compact", "lg_h2o_reset", "lg_h2o_evict", "lg_read_device_status",
            "lg_decode_attend_noalloc", "lg_detect_state_size", "lg_streaming_evict",
            "lg_detect_prune", "lg_default_token_params", "lg_token_state_size",
            "lg_token_detect", "lg_token_detect_prune"]



def chunk_symbols():
    """names of the C ABI functions declared in include/lg_chunk.h"""
    return ["lg_begin_chunk", "lg_default_rope_params", "lg_rope_append",
            "lg_chunk_workspace_size", "lg_chunk_attend", "lg_count_tokens", "lg_pick_token"]


def draft_symbols():
    """names of the C ABI functions declared in include/lg_draft.h"""
    return ["lg_verify_workspace_size", "lg_verify_draft", "lg_end_chunk", "lg_read_rows"]


NOALLOC_SCRATCH_BYTES = 32 << 20  # LG_NOALLOC_SCRATCH_BYTES in include/lg.h


def _ptr(t):
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


# The current stream's handle without building a torch.cuda.Stream around it: 2.8 us of the
# 8.9 us a lg_decode_attend call took its caller (Grace), more than the launch itself.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _get_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_get_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _call(name, *args):
    rc = getattr(_lib or lib(), name)(*args)
    if rc != LG_OK:
        raise LgError(name, rc)


# ------------------------------------------------------------------ thin wrappers, same names

def lg_default_params(**over) -> LgGuardParams:
    p = LgGuardParams()
    _call("lg_default_params", ctypes.byref(p))
    for k, v in over.items():
        setattr(p, k, v)
    return p


def lg_status_string(code: int) -> str:
    return lib().lg_status_string(code).decode()


def lg_workspace_size(cache, H_q, n_layers, max_len, accumulate_h2o=0) -> int:
    return int(lib().lg_workspace_size(ctypes.byref(cache.c), H_q, n_layers, max_len,
                                       accumulate_h2o))


def lg_state_init(cache, state, t_gen0=64, stream=None):
    _call("lg_state_init", ctypes.byref(cache.c), _ptr(state), t_gen0, _stream(stream))


def lg_begin_step(cache, stream=None):
    _call("lg_begin_step", ctypes.byref(cache.c), _stream(stream))


def lg_append(cache, layer0, n_layers, k_new, v_new, pos_new, params, stream=None):
    _call("lg_append", ctypes.byref(cache.c), layer0, n_layers, _ptr(k_new), _ptr(v_new),
          _ptr(pos_new), ctypes.byref(params), _stream(stream))


def lg_sketch_build(cache, params, max_len, stream=None):
    _call("lg_sketch_build", ctypes.byref(cache.c), ctypes.byref(params), max_len,
          _stream(stream))


def lg_decode_attend(cache, layer0, n_layers, q, H_q, scale, out, stats, suffix_w,
                     accumulate_h2o, max_len, ws, stream=None):
    _call("lg_decode_attend", ctypes.byref(cache.c), layer0, n_layers, _ptr(q), H_q,
          float(scale), _ptr(out), _ptr(stats), suffix_w, accumulate_h2o, max_len, _ptr(ws),
          ws.numel() * ws.element_size(), _stream(stream))


def lg_decode_attend_noalloc(cache, layer0, n_layers, q, H_q, scale, out, stats, suffix_w,
                             accumulate_h2o, max_len, stream=None):
    """lg_decode_attend with the library's own static scratch (no workspace argument)"""
    _call("lg_decode_attend_noalloc", ctypes.byref(cache.c), layer0, n_layers, _ptr(q), H_q,
          float(scale), _ptr(out), _ptr(stats), suffix_w, accumulate_h2o, max_len,
          _stream(stream))


def lg_detect_state_size(cache, params) -> int:
    return int(lib().lg_detect_state_size(ctypes.byref(cache.c), ctypes.byref(params)))


def lg_default_token_params(**over) -> LgTokenParams:
    tp = LgTokenParams()
    _call("lg_default_token_params", ctypes.byref(tp))
    for k, v in over.items():
        setattr(tp, k, v)
    return tp


def lg_token_state_size(cache, params, tparams) -> int:
    return int(lib().lg_token_state_size(ctypes.byref(cache.c), ctypes.byref(params),
                                         ctypes.byref(tparams)))


def lg_token_detect(cache, tokens, pmax, state, params, tparams, flags, spans, diag, tstate,
                    kept_idx=None, kept_count=None, stream=None):
    """kept_idx / kept_count: the buffers lg_prune_compact wrote after the previous call (or
    None): the trailing kept rows that are still consecutive tokens keep mapping the span"""
    max_keep = int(kept_idx.shape[1]) if kept_idx is not None else 0
    _call("lg_token_detect", ctypes.byref(cache.c), _ptr(tokens), _ptr(pmax), _ptr(kept_idx),
          _ptr(kept_count), max_keep, _ptr(state), ctypes.byref(params), ctypes.byref(tparams),
          _ptr(flags), _ptr(spans), _ptr(diag), _ptr(tstate), _stream(stream))


def lg_token_detect_prune(cache, tokens, pmax, state, budget, params, tparams, flags, spans,
                          diag, tstate, kept_idx, kept_count, max_keep, max_len, stream=None):
    """lg_token_detect then lg_prune_compact in two launches; kept_idx / kept_count carry the
    previous prune's lists in and this step's out"""
    _call("lg_token_detect_prune", ctypes.byref(cache.c), _ptr(tokens), _ptr(pmax), _ptr(state),
          _ptr(budget), ctypes.byref(params), ctypes.byref(tparams), _ptr(flags), _ptr(spans),
          _ptr(diag), _ptr(tstate), _ptr(kept_idx), _ptr(kept_count), max_keep, max_len,
          _stream(stream))


def lg_detect(cache, stats, H_q, state, budget, params, flags, spans, diag, dstate, stream=None):
    _call("lg_detect", ctypes.byref(cache.c), _ptr(stats), H_q, _ptr(state), _ptr(budget),
          ctypes.byref(params), _ptr(flags), _ptr(spans), _ptr(diag), _ptr(dstate),
          _stream(stream))


def lg_detect_prune(cache, stats, H_q, state, budget, params, flags, spans, diag, dstate,
                    kept_idx, kept_count, max_keep, max_len, stream=None):
    _call("lg_detect_prune", ctypes.byref(cache.c), _ptr(stats), H_q, _ptr(state), _ptr(budget),
          ctypes.byref(params), _ptr(flags), _ptr(spans), _ptr(diag), _ptr(dstate),
          _ptr(kept_idx), _ptr(kept_count), max_keep, max_len, _stream(stream))


def lg_prune_compact(cache, flags, spans, state, budget, params, kept_idx, kept_count, max_keep,
                     max_len, stream=None):
    _call("lg_prune_compact", ctypes.byref(cache.c), _ptr(flags), _ptr(spans), _ptr(state),
          _ptr(budget), ctypes.byref(params), _ptr(kept_idx), _ptr(kept_count), max_keep,
          max_len, _stream(stream))


def lg_h2o_reset(cache, max_len, stream=None):
    _call("lg_h2o_reset", ctypes.byref(cache.c), max_len, _stream(stream))


def lg_h2o_evict(cache, budget, pos_now, max_len, stream=None):
    _call("lg_h2o_evict", ctypes.byref(cache.c), _ptr(budget), _ptr(pos_now), max_len,
          _stream(stream))


def lg_streaming_evict(cache, budget, pos_now, n_sink, max_len, stream=None):
    _call("lg_streaming_evict", ctypes.byref(cache.c), _ptr(budget), _ptr(pos_now), n_sink,
          max_len, _stream(stream))


N_SINK = 4  # StreamingLLM attention sinks (count not stated by the paper)


def lg_read_device_status(cache, stream=None) -> int:
    code = ctypes.c_int32(0)
    _call("lg_read_device_status", ctypes.byref(cache.c), ctypes.byref(code), _stream(stream))
    return code.value


# ------------------------------------------------------------------ chunks and picked tokens

class Chunk:
    """The new tokens of a batch (lg_chunk): off, int32 device tensor [batch + 1]; T, rows of the
    token arrays; max_new, a bound on the new tokens of one sequence."""

    def __init__(self, off, T, max_new):
        if off.dtype is not torch.int32 or not off.is_contiguous():
            raise ValueError("off: dense [batch + 1] int32")
        self.off, self.T, self.max_new = off, int(T), int(max_new)
        self.c = LgChunk(off=_ptr(off), T=self.T, max_new=self.max_new)

    @classmethod
    def of(cls, counts, device):
        """the chunk of counts[b] new tokens of each sequence, rows one after another"""
        off = np.concatenate([[0], np.cumsum(np.asarray(counts, dtype=np.int64))])
        return cls(torch.as_tensor(off.astype(np.int32), device=device), int(off[-1]),
                   int(max(counts)))


def _rows_stride(t, name, T=0, H=0, d=0):
    """elements from token to token of a [T][H][d] tensor whose rows are whole (T rows and H heads at
    least)"""
    if t.dim() != 3:
        raise ValueError("%s: [T][H][d]" % name)
    n, h, e = t.shape
    step, head, one = t.stride()
    if one != 1 or head != e and h > 1 or n < T or h < H or e != d and d:
        raise ValueError("%s: [T][H][d] with whole rows of H * d elements" % name)
    row = h * e
    if n == 1:  # its stride says nothing
        return row
    if step < row:  # one row for every token, for instance
        raise ValueError("%s: [T][H][d] with rows that do not overlap" % name)
    return step


# The calls below refuse what their kernels could not read: tensors of another type, too short, not
# dense (a slice, one row expanded over the batch), or of another device than the current one, whose
# stream the call takes.
def _refuse(what, needs):
    raise ValueError("%s: on the current CUDA device, dense, %s" % (what, needs))


def _dense(t, dt, n, at):
    """n elements of the type dt at t's address, at least, on device `at`"""
    return t.dtype is dt and t.numel() >= n and t.is_contiguous() and t.get_device() == at


def _dense_rows(t, dt, rows, cols, at):
    """the same of rows of cols, as a matrix of them or flat; dt None: any words of 32 bits"""
    sh = t.shape
    return ((t.element_size() == 4 if dt is None else t.dtype is dt) and t.is_contiguous() and
            t.get_device() == at and
            (sh[0] >= rows and sh[1] == cols if len(sh) == 2 else t.numel() >= rows * cols))


_device = _get_device or torch.cuda.current_device


def _device_of(cache, chunk):
    """the current device, which the cache and the chunk's offsets are on"""
    at, off = _device(), chunk.off
    if cache.status.get_device() != at:
        _refuse("cache", "its buffers")
    if off.numel() <= cache.c.batch or off.get_device() != at:
        _refuse("off", "[batch + 1] int32")
    return at


def _row_type(cache):
    """the type of queries, new rows and results: the cache's, bf16 for one of four bits"""
    dt = cache.k.dtype
    return torch.bfloat16 if dt is torch.uint8 else dt


def lg_begin_chunk(cache, chunk, stream=None):
    _device_of(cache, chunk)
    _call("lg_begin_chunk", ctypes.byref(cache.c), ctypes.byref(chunk.c), _stream(stream))


def lg_default_rope_params(d, **over) -> LgRopeParams:
    p = LgRopeParams()
    _call("lg_default_rope_params", ctypes.byref(p), d)
    for k, v in over.items():
        setattr(p, k, v)
    return p


def lg_rope_append(cache, chunk, layer, q, k_new, v_new, pos, rope, q_out, params, stream=None):
    """q [T][H_q][d] (or None with q_out None), k_new, v_new [T][H_kv][d]: slices of one packed
    projection pass as they are"""
    if q_out is not None and not q_out.is_contiguous():
        raise ValueError("q_out: dense [T][H_q][d]")
    T, H_kv, d, dt = chunk.T, cache.H_kv, cache.d, _row_type(cache)
    at = _device_of(cache, chunk)
    H_q = qs = 0
    if q is not None:
        H_q, qs = q.shape[1], _rows_stride(q, "q", T, 0, d)
        if q.dtype is not dt or q.get_device() != at:
            _refuse("q", "[T][H_q][d] of the cache's type")
    if q_out is not None and (q_out.dtype is not dt or q_out.numel() < T * H_q * d or
                              q_out.get_device() != at):
        _refuse("q_out", "[T][H_q][d] of the cache's type")
    ks, vs = _rows_stride(k_new, "k_new", T, H_kv, d), _rows_stride(v_new, "v_new", T, H_kv, d)
    if (k_new.dtype is not dt or v_new.dtype is not dt or k_new.get_device() != at or
            v_new.get_device() != at):
        _refuse("k_new, v_new", "[T][H_kv][d] of the cache's type")
    if pos is not None and not _dense(pos, torch.int32, T, at):
        _refuse("pos", "[T] int32")
    rc = (_lib or lib()).lg_rope_append(
        ctypes.byref(cache.c), ctypes.byref(chunk.c), layer, None if q is None else q.data_ptr(), qs,
        H_q, k_new.data_ptr(), ks, v_new.data_ptr(), vs, None if pos is None else pos.data_ptr(),
        ctypes.byref(rope), None if q_out is None else q_out.data_ptr(),
        ctypes.byref(params), _raw_stream(at) if stream is None and _raw_stream else _stream(stream))
    if rc:
        raise LgError("lg_rope_append", rc)


def lg_chunk_workspace_size(cache, chunk, H_q, max_len) -> int:
    return int(lib().lg_chunk_workspace_size(ctypes.byref(cache.c), ctypes.byref(chunk.c), H_q,
                                             max_len))


def lg_chunk_attend(cache, chunk, layer, q, H_q, scale, window, n_sink, out, max_len, ws,
                    stream=None):
    if not (q.is_contiguous() and out.is_contiguous()):
        raise ValueError("q, out: dense [T][H_q][d]")
    n, dt, at = chunk.T * H_q * cache.d, _row_type(cache), _device_of(cache, chunk)
    if (q.dtype is not dt or out.dtype is not dt or q.numel() < n or out.numel() < n or
            q.get_device() != at or out.get_device() != at):
        _refuse("q, out", "[T][H_q][d] of the cache's type")
    if not ws.is_contiguous() or ws.get_device() != at:
        _refuse("ws", "bytes")
    rc = (_lib or lib()).lg_chunk_attend(
        ctypes.byref(cache.c), ctypes.byref(chunk.c), layer, q.data_ptr(), H_q,
        float(scale), window, n_sink, out.data_ptr(), max_len, ws.data_ptr(), ws.nbytes,
        _raw_stream(at) if stream is None and _raw_stream else _stream(stream))
    if rc:
        raise LgError("lg_chunk_attend", rc)


def lg_count_tokens(tokens, off, V, generated, seen, counts, status=None, stream=None):
    """tokens of row b: tokens[off[b]] .. tokens[off[b + 1] - 1], or tokens[b] with off None"""
    batch = tokens.numel() if off is None else off.numel() - 1
    at = _device()
    if (not _dense(tokens, torch.int32, 0, at) or
            not _dense_rows(counts, torch.int32, batch, V, at) or
            not _dense_rows(seen, None, batch, (V + 31) // 32, at)):
        _refuse("tokens, seen, counts", "int32, [batch][ceil(V/32)] words, [batch][V] int32")
    if off is not None and not _dense(off, torch.int32, 0, at):
        _refuse("off", "[batch + 1] int32")
    if status is not None and not _dense(status, torch.int32, 1, at):
        _refuse("status", "a word of int32")
    _call("lg_count_tokens", _ptr(tokens), _ptr(off), tokens.numel(), batch, V, generated,
          _ptr(seen), _ptr(counts), _ptr(status), _stream(stream))


_I32, _F32, _BF16 = torch.int32, torch.float32, torch.bfloat16
_lg_logits = struct.Struct("@Piiiiq").pack  # an lg_logits, in a quarter of the structure's time
_LOGITS = {torch.bfloat16: LG_BF16, torch.float32: LG_F32}


def lg_pick_token(logits, seen, counts, penalty, bias, allowed, tokens, pmax, status=None,
                  logits_out=None, stream=None):
    """logits [batch][V] (rows may be strided); bias: None or (off, id, val); status: the cache's
    status word or None; logits_out: None or a tensor of the same dtype and strides"""
    st = logits.stride()
    if len(st) != 2 or st[1] != 1:
        raise ValueError("logits: [batch][V] with whole rows")
    B, V = logits.shape
    if B > 1 and st[0] < V:
        raise ValueError("logits: [batch][V] with rows that do not overlap")
    if logits_out is not None and (logits_out.dtype is not logits.dtype or
                                   logits_out.stride() != st or logits_out.shape != (B, V)):
        raise ValueError("logits_out: dtype, strides and shape of logits")
    at = _device()
    if logits.get_device() != at or logits_out is not None and logits_out.get_device() != at:
        _refuse("logits, logits_out", "[batch][V]")
    nw = (V + 31) // 32
    # (in place what _dense and _dense_rows ask, of the tensors of every step: a row's call is as long
    # on the host as on the GPU; through the functions pick_one took 7.7 us, not 6.9)
    if not (tokens.dtype is _I32 and tokens.numel() >= B and tokens.is_contiguous() and
            tokens.get_device() == at and pmax.dtype is _F32 and pmax.numel() >= B and
            pmax.is_contiguous() and pmax.get_device() == at):
        _refuse("tokens, pmax", "[batch] int32, fp32")
    if seen is not None:
        sh = seen.shape
        if not (seen.element_size() == 4 and seen.is_contiguous() and seen.get_device() == at and
                (sh[0] >= B and sh[1] == nw if len(sh) == 2 else seen.numel() >= B * nw)):
            _refuse("seen", "[batch][ceil(V/32)] words")
    if counts is not None:
        sh = counts.shape
        if not (counts.dtype is _I32 and counts.is_contiguous() and counts.get_device() == at and
                (sh[0] >= B and sh[1] == V if len(sh) == 2 else counts.numel() >= B * V)):
            _refuse("counts", "[batch][V] int32")
    if penalty is not None:
        sh = penalty.shape
        if not (penalty.dtype is _F32 and penalty.is_contiguous() and penalty.get_device() == at and
                (sh[0] >= B and sh[1] == 4 if len(sh) == 2 else penalty.numel() >= 4 * B)):
            _refuse("penalty", "[batch][4] fp32")
    if status is not None and not (status.dtype is _I32 and status.get_device() == at and
                                   status.numel()):
        _refuse("status", "a word of int32")
    if allowed is not None and not _dense_rows(allowed, None, B, nw, at):
        _refuse("allowed", "[batch][ceil(V/32)] words")
    bs = None
    if bias is not None:
        off, ids, val = bias
        if (not _dense(off, torch.int32, B + 1, at) or not _dense(ids, torch.int32, 0, at) or
                not _dense(val, torch.float32, ids.numel(), at)):
            _refuse("bias", "[batch + 1] int32, int32, as many fp32")
        bs = ctypes.byref(LgBias(off.data_ptr(), ids.data_ptr(), val.data_ptr()))
    x = _lg_logits(logits.data_ptr(), _LOGITS.get(logits.dtype, -1), B, V, 0,
                   st[0] if B > 1 else V)  # one row: its stride says nothing
    rc = (_lib or lib()).lg_pick_token(
        x, None if seen is None else seen.data_ptr(),
        None if counts is None else counts.data_ptr(),
        None if penalty is None else penalty.data_ptr(), bs,
        None if allowed is None else allowed.data_ptr(), tokens.data_ptr(), pmax.data_ptr(),
        None if logits_out is None else logits_out.data_ptr(),
        None if status is None else status.data_ptr(),
        _raw_stream(at) if stream is None and _raw_stream else _stream(stream))
    if rc:
        raise LgError("lg_pick_token", rc)


# ------------------------------------------------------------------ drafted tokens, 4-bit rows

def _logits_of(t, name):
    """an lg_logits of [rows][V] with whole rows that do not overlap"""
    sh, st = t.shape, t.stride()
    if len(sh) != 2 or st[1] != 1 or sh[0] > 1 and st[0] < sh[1]:
        raise ValueError("%s: [T][V] with whole rows that do not overlap" % name)
    B, V = sh
    return _lg_logits(t.data_ptr(), _LOGITS.get(t.dtype, -1), B, V, 0, st[0] if B > 1 else V)


def lg_verify_workspace_size(logits, chunk) -> int:
    return int(lib().lg_verify_workspace_size(_logits_of(logits, "logits"), ctypes.byref(chunk.c)))


def lg_verify_draft(logits, chunk, tokens, draft, temperature, u, r, picked, accepted, ws,
                    status=None, stream=None):
    """logits [T][V], row t the target's after tokens[t]; draft: probabilities [T][V] (its own type and
    stride) or None; temperature [batch] or None, u [T], r [batch] fp32; picked [T], accepted [batch]
    int32; ws: lg_verify_workspace_size bytes"""
    off = chunk.off
    T, batch, at = chunk.T, off.numel() - 1, _device()
    x = _logits_of(logits, "logits")
    y = None if draft is None else _logits_of(draft, "draft")
    if off.get_device() != at:
        _refuse("off", "[batch + 1] int32")
    if logits.get_device() != at or draft is not None and draft.get_device() != at:
        _refuse("logits, draft", "[T][V]")
    # (in place what _dense asks, as in lg_pick_token)
    if not (tokens.dtype is _I32 and tokens.numel() >= T and tokens.is_contiguous() and
            tokens.get_device() == at and picked.dtype is _I32 and picked.numel() >= T and
            picked.is_contiguous() and picked.get_device() == at and accepted.dtype is _I32 and
            accepted.numel() >= batch and accepted.is_contiguous() and accepted.get_device() == at):
        _refuse("tokens, picked, accepted", "[T], [T], [batch] int32")
    if not (u.dtype is _F32 and u.numel() >= T and u.is_contiguous() and u.get_device() == at and
            r.dtype is _F32 and r.numel() >= batch and r.is_contiguous() and r.get_device() == at and
            (temperature is None or _dense(temperature, _F32, batch, at))):
        _refuse("u, r, temperature", "[T], [batch], [batch] fp32")
    if status is not None and not _dense(status, _I32, 1, at):
        _refuse("status", "a word of int32")
    if not ws.is_contiguous() or ws.get_device() != at:
        _refuse("ws", "bytes")
    rc = (_lib or lib()).lg_verify_draft(
        x, ctypes.byref(chunk.c), batch, tokens.data_ptr(), y,
        None if temperature is None else temperature.data_ptr(), u.data_ptr(), r.data_ptr(),
        picked.data_ptr(), accepted.data_ptr(), ws.data_ptr(), ws.nbytes,
        None if status is None else status.data_ptr(),
        _raw_stream(at) if stream is None and _raw_stream else _stream(stream))
    if rc:
        raise LgError("lg_verify_draft", rc)


def lg_end_chunk(cache, chunk, accepted, stream=None):
    at = _device_of(cache, chunk)
    if not _dense(accepted, _I32, cache.c.batch, at):
        _refuse("accepted", "[batch] int32")
    _call("lg_end_chunk", ctypes.byref(cache.c), ctypes.byref(chunk.c), _ptr(accepted),
          _stream(stream))


def lg_read_rows(cache, chunk, layer, k_out, v_out, stream=None):
    """the chunk's rows of a 4-bit cache as values: k_out, v_out [T][H_kv][d] bf16"""
    n, at = chunk.T * cache.H_kv * cache.d, _device_of(cache, chunk)
    if not (k_out.dtype is _BF16 and k_out.numel() >= n and k_out.is_contiguous() and
            k_out.get_device() == at and v_out.dtype is _BF16 and v_out.numel() >= n and
            v_out.is_contiguous() and v_out.get_device() == at):
        _refuse("k_out, v_out", "[T][H_kv][d] bf16")
    rc = (_lib or lib()).lg_read_rows(
        ctypes.byref(cache.c), ctypes.byref(chunk.c), layer, k_out.data_ptr(), v_out.data_ptr(),
        _raw_stream(at) if stream is None and _raw_stream else _stream(stream))
    if rc:
        raise LgError("lg_read_rows", rc)


# ------------------------------------------------------------------ device buffers of a batch

def _torch_dtype(dtype: str):
    """of queries, new rows and results"""
    return torch.float32 if dtype == "f32" else torch.bfloat16


_DTYPES = {"bf16": LG_BF16, "f32": LG_F32, "q4": LG_Q4}


def host_to_device(a: np.ndarray, device, dtype: str):
    """numpy cache-dtype array (bf16 as uint16 bits, or float32) -> torch tensor on device"""
    if dtype != "f32":
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(
            torch.bfloat16).to(device)
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)


def device_to_host(t: torch.Tensor) -> np.ndarray:
    t = t.detach().cpu()
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).numpy().view(np.uint16)
    return t.numpy()


class Cache:
    """Device KV cache of a batch laid out as lg_cache documents, plus its metadata.
    policy 'loopguard' allocates sketches; 'h2o' allocates scores and positions.  dtype 'bf16', 'f32' or
    'q4': rows in four bits, k and v then bytes [L][H_kv][S_total][d/2 + 16] (LG_Q4 of lg.h)."""

    def __init__(self, L, H_kv, d, dtype, seq_off, cap, n0, device, policy="loopguard",
                 k=None, v=None):
        self.L, self.H_kv, self.d, self.dtype = L, H_kv, d, dtype
        self.device = torch.device(device)
        self.batch = len(cap)
        self.S_total = int(np.asarray(cap, dtype=np.int64).sum())
        if dtype == "q4" and policy not in ("loopguard", "none"):
            raise ValueError("a cache of four bits has no scores and positions")
        tdt = torch.uint8 if dtype == "q4" else _torch_dtype(dtype)
        shape = (L, H_kv, self.S_total, d // 2 + 16 if dtype == "q4" else d)
        self.k = k if k is not None else torch.zeros(shape, dtype=tdt, device=self.device)
        self.v = v if v is not None else torch.zeros(shape, dtype=tdt, device=self.device)
        self.seq_off = torch.as_tensor(np.asarray(seq_off, dtype=np.int64), device=self.device)
        self.cap = torch.as_tensor(np.asarray(cap, dtype=np.int32), device=self.device)
        self.len = torch.as_tensor(np.asarray(n0, dtype=np.int32), device=self.device).clone()
        self.nwords = H_kv * d // 32
        self.sketch = None
        self.h2o = self.pos = None
        if policy == "loopguard":
            self.sketch = torch.zeros((self.S_total, self.nwords), dtype=torch.int32,
                                      device=self.device)
        if policy in ("h2o", "streaming", "full"):
            self.h2o = torch.zeros((L, H_kv, self.S_total), dtype=torch.float32,
                                   device=self.device)
            self.pos = torch.zeros((L, H_kv, self.S_total), dtype=torch.int32,
                                   device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.c = LgCache(k=_ptr(self.k), v=_ptr(self.v), dtype=_DTYPES[dtype], L=L, H_kv=H_kv, d=d, batch=self.batch, pad=0,
                         S_total=self.S_total, seq_off=_ptr(self.seq_off), cap=_ptr(self.cap),
                         len=_ptr(self.len), sketch=_ptr(self.sketch), h2o=_ptr(self.h2o),
                         pos=_ptr(self.pos), dev_status=_ptr(self.status))

    @classmethod
    def from_host(cls, w, K, V, device, policy="loopguard", params=None):
        """cache of workload w from host arrays K, V [L][H_kv][S_total][d] (rows [0, n0))"""
        k = host_to_device(K, device, w.dtype)
        v = host_to_device(V, device, w.dtype)
        c = cls(w.L, w.H_kv, w.d, w.dtype, w.seq_off, w.cap, w.n0, device, policy, k, v)
        c.prepare(int(w.n0.max()), params)
        return c

    def prepare(self, max_len, params=None):
        """after a prefill: sketches of the guard layer, or H2O positions and scores (a cache of four
        bits has its sketches from the appends)"""
        if self.sketch is not None and self.dtype != "q4":
            lg_sketch_build(self, params or lg_default_params(), max_len)
        if self.h2o is not None:
            lg_h2o_reset(self, max_len)

    def to_host(self):
        return device_to_host(self.k), device_to_host(self.v)

    def lengths(self) -> np.ndarray:
        return self.len.cpu().numpy()


class Guard:
    """Device buffers and call order of one guarded decode step (lg.h) for a Cache."""

    def __init__(self, cache: Cache, H_q: int, params: LgGuardParams | None = None,
                 policy="loopguard", max_len=None, t_gen0=64, n_layers_per_call=None,
                 fused_prune=True):
        self.cache = cache
        self.fused_prune = fused_prune  # lg_detect_prune, else lg_detect + lg_prune_compact
        self.H_q = H_q
        self.p = params or lg_default_params()
        self.policy = policy
        dev = cache.device
        cap = cache.cap.cpu().numpy()
        self.max_len = int(cap.max()) if max_len is None else int(max_len)
        self.max_keep = self.max_len
        self.n_layers_per_call = n_layers_per_call or cache.L
        L, b = cache.L, cache.batch
        self.state = torch.zeros((b, STATE_BYTES // 4), dtype=torch.int32, device=dev)
        # flags and spans side by side (one read-back of a step's decisions)
        self.flags_spans = torch.zeros(3 * b, dtype=torch.int32, device=dev)
        self.flags = self.flags_spans[:b]
        self.spans = self.flags_spans[b:].view(b, 2)
        self.kept_idx = torch.zeros((b, self.max_keep), dtype=torch.int32, device=dev)
        self.kept_count = torch.zeros(b, dtype=torch.int32, device=dev)
        self.diag = torch.zeros((b, 8), dtype=torch.float64, device=dev)
        ds_words = lg_detect_state_size(cache, self.p) // 4 if policy == "loopguard" else 1
        self.dstate = torch.zeros(ds_words, dtype=torch.int32, device=dev)
        tdt = _torch_dtype(cache.dtype)
        self.out = torch.zeros((L, b, H_q, cache.d), dtype=tdt, device=dev)
        self.stats = torch.zeros((L, b, H_q, 4), dtype=torch.float32, device=dev)
        h2o = 1 if policy == "h2o" else 0
        ws_bytes = lg_workspace_size(cache, H_q, self.n_layers_per_call, self.max_len, h2o)
        self.ws = torch.empty(ws_bytes // 4 + 64, dtype=torch.float32, device=dev)
        self.scale = 1.0 / float(np.sqrt(cache.d))
        lg_state_init(cache, self.state, t_gen0)

    def step(self, q, k_new, v_new, budget, pos_new=None, stream=None):
        """one guarded decode step on device tensors:
        q [L][b][H_q][d], k_new/v_new [L][b][H_kv][d], budget [b] int32, pos_new [b] int32"""
        c, p = self.cache, self.p
        lg_begin_step(c, stream)
        lg_append(c, 0, c.L, k_new, v_new, pos_new, p, stream)
        for l0 in range(0, c.L, self.n_layers_per_call):
            nl = min(self.n_layers_per_call, c.L - l0)   # the last call takes what is left
            lg_decode_attend(c, l0, nl, q[l0:l0 + nl], self.H_q, self.scale, self.out[l0:l0 + nl],
                             self.stats[l0:l0 + nl], p.suffix_w, 1 if self.policy == "h2o" else 0,
                             self.max_len, self.ws, stream)
        if self.policy == "loopguard" and self.fused_prune:
            lg_detect_prune(c, self.stats, self.H_q, self.state, budget, p, self.flags,
                            self.spans, self.diag, self.dstate, self.kept_idx, self.kept_count,
                            self.max_keep, self.max_len, stream)
        elif self.policy == "loopguard":
            lg_detect(c, self.stats, self.H_q, self.state, budget, p, self.flags, self.spans,
                      self.diag, self.dstate, stream)
            lg_prune_compact(c, self.flags, self.spans, self.state, budget, p, self.kept_idx,
                             self.kept_count, self.max_keep, self.max_len, stream)
        elif self.policy == "h2o":
            lg_h2o_evict(c, budget, pos_new, self.max_len, stream)
        elif self.policy == "streaming":
            lg_streaming_evict(c, budget, pos_new, N_SINK, self.max_len, stream)

    def step_host(self, q, k_new, v_new, budget, pos_new=None):
        """same step from host numpy arrays; returns host copies of every output"""
        dev, dt = self.cache.device, self.cache.dtype
        qd = host_to_device(q, dev, dt)
        kd = host_to_device(k_new, dev, dt)
        vd = host_to_device(v_new, dev, dt)
        bd = torch.as_tensor(np.asarray(budget, dtype=np.int32), device=dev)
        pd = None if pos_new is None else torch.as_tensor(np.asarray(pos_new, dtype=np.int32),
                                                          device=dev)
        self.step(qd, kd, vd, bd, pd)
        return self.results()

    def results(self):
        torch.cuda.current_stream().synchronize()
        st = lg_read_device_status(self.cache)
        if st != 0:
            raise LgError("device status", st)
        r = dict(out=device_to_host(self.out).astype(np.float32) if self.cache.dtype == "f32"
                 else (device_to_host(self.out).astype(np.uint32) << 16).view(np.float32),
                 stats=self.stats.cpu().numpy(), len=self.cache.lengths())
        if self.policy == "loopguard":
            r.update(flags=self.flags.cpu().numpy(), spans=self.spans.cpu().numpy(),
                     kept_count=self.kept_count.cpu().numpy(),
                     kept_idx=self.kept_idx.cpu().numpy(),
                     state=self.state.cpu().numpy(), diag=self.diag.cpu().numpy())
        return r
