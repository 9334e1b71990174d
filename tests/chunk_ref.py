"""Plain 64-bit forms of the calls of include/lg_chunk.h, and batches to run them on.

Tolerances of the attention, from its roundings (A = sum_i a_i |v_i|, the weights applied to
absolute values):
  bf16: the weights reach the matrix product rounded to bf16 (2^-8 of each at most), the result is
        rounded once (2^-8 of it); scores, exponentials and sums in fp32 stay below 2^-12:
        |d| <= 2^-8 |ref| + (2^-8 + 2^-12) A
  fp32: a score is a sum of d products, off by at most (d + 4) 2^-24 sum_e |q_e k_e| scale (z below
        is the largest such sum); a weight by that twice (numerator and normaliser), by 2^-21 for
        the exponentials and by n 2^-24 for the sums of n terms:
        |d| <= 2^-24 |ref| + (2 (d + 4) 2^-24 z + 2^-20 + 2 n 2^-24) A
"""
import math

import numpy as np
import torch

from paper_2604_10044_gb300 import lg


def tdtype(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class Batch:
    """A cache of layers [0, L) whose sequences hold ns[b] rows, ms[b] of them new, with queries;
    gaps of two slots between sequences.  Everything outside the rows is NaN."""

    def __init__(self, ns, ms, dtype="bf16", H_kv=2, g=4, d=128, L=1, seed=0, device="cuda:0",
                 spread=1.0, pad_rows=3, policy="loopguard"):
        self.ns, self.ms, self.dtype, self.H_kv, self.g, self.d = ns, ms, dtype, H_kv, g, d
        self.H_q = H_kv * g
        gen = torch.Generator().manual_seed(seed)
        cap = np.array([n + 2 for n in ns], dtype=np.int32)
        self.seq = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
        S = int(cap.sum())
        dt = tdtype(dtype)
        self.k = torch.full((L, H_kv, S, d), math.nan, dtype=dt)
        self.v = torch.full((L, H_kv, S, d), math.nan, dtype=dt)
        for o, n in zip(self.seq, ns):
            self.k[:, :, o:o + n] = (torch.randn((L, H_kv, n, d), generator=gen) * spread).to(dt)
            self.v[:, :, o:o + n] = torch.randn((L, H_kv, n, d), generator=gen).to(dt)
        self.T = sum(ms) + pad_rows          # rows behind the last sequence
        self.q = torch.full((self.T, self.H_q, d), math.nan, dtype=dt)
        self.q[:sum(ms)] = torch.randn((sum(ms), self.H_q, d), generator=gen).to(dt)
        self.cap, self.L, self.policy, self.device = cap, L, policy, device

    def to_device(self):
        dev = self.device
        self.cache = lg.Cache(self.L, self.H_kv, self.d, self.dtype, self.seq, self.cap,
                              np.array(self.ns, dtype=np.int32), dev, self.policy,
                              self.k.to(dev), self.v.to(dev))
        ch = lg.Chunk.of(self.ms, dev)
        self.chunk = lg.Chunk(ch.off, self.T, ch.max_new)
        self.qd = self.q.to(dev)
        self.max_len = max(max(self.ns), 1)
        n = lg.lg_chunk_workspace_size(self.cache, self.chunk, self.H_q, self.max_len)
        assert n > 0 and n % 256 == 0
        self.ws = torch.full((n,), 0xff, dtype=torch.uint8, device=dev)  # NaN words
        return self

    def attend(self, window=0, sink=0, layer=0, stream=None):
        """the call's output, rows it may not write still 7"""
        out = torch.full_like(self.qd, 7.0)
        lg.lg_chunk_attend(self.cache, self.chunk, layer, self.qd, self.H_q, self.d ** -0.5,
                           window, sink, out, self.max_len, self.ws, stream)
        return out

    def reference(self, window=0, sink=0, layer=0):
        """(ref, tol) of every query row in 64 bits, NaN-free hidden rows or not"""
        ref = torch.full((self.T, self.H_q, self.d), 7.0, dtype=torch.float64)
        tol = torch.zeros_like(ref)
        t = 0
        for o, n, m in zip(self.seq, self.ns, self.ms):
            for h in range(self.H_q if m else 0):
                K = self.k[layer, h // self.g, o:o + n].double()
                V = self.v[layer, h // self.g, o:o + n].double()
                Q = self.q[t:t + m, h].double()
                see = visible(n, m, window, sink)
                s = torch.where(see, Q @ K.T * self.d ** -0.5, -math.inf)
                a = torch.softmax(s, -1)
                V0 = torch.nan_to_num(V, nan=0.0, posinf=0.0, neginf=0.0)
                ref[t:t + m, h] = a @ V0
                # a row that sees something that is not a number has no number either
                for i in torch.nonzero(~torch.isfinite(V).all(-1))[:, 0].tolist():
                    x = torch.where(torch.isfinite(V[i]), 0.0, V[i])
                    ref[t:t + m, h] += torch.where(see[:, i:i + 1], x, 0.0)
                A = a @ V0.abs()
                if self.dtype == "bf16":
                    tol[t:t + m, h] = 2.0 ** -8 * ref[t:t + m, h].abs() + (2.0 ** -8 + 2.0 ** -12) * A
                else:
                    z = torch.nan_to_num(Q.abs() @ K.abs().T).max() * self.d ** -0.5
                    w = 2 * (self.d + 4) * 2.0 ** -24 * z + 2.0 ** -20 + 2 * n * 2.0 ** -24
                    tol[t:t + m, h] = 2.0 ** -24 * ref[t:t + m, h].abs() + w * A
            t += m
        return ref, tol

    def check(self, out, window=0, sink=0, layer=0):
        assert lg.lg_read_device_status(self.cache) == 0
        ref, tol = self.reference(window, sink, layer)
        got = out.double().cpu()
        assert (got[sum(self.ms):] == 7.0).all(), "rows behind the last sequence"
        bad = (got - ref).abs() > tol
        bad |= torch.isnan(got) != torch.isnan(ref)
        bad &= ~(torch.isinf(ref) & (got == ref))
        if bad.any():
            i = tuple(torch.nonzero(bad)[0].tolist())
            raise AssertionError("%d of %d outside, first at %s: %r, want %r (tol %r)" % (
                int(bad.sum()), bad.numel(), i, got[i].item(), ref[i].item(), tol[i].item()))


def visible(n, m, window, sink):
    """[m][n]: what each new row sees"""
    r = torch.arange(n - m, n)[:, None]
    i = torch.arange(n)[None]
    see = i <= r
    if window:
        see &= (i > r - window) | (i < sink)
    return see


def frequencies(p, d):
    """radians a position, from the documented formulas"""
    rot, theta = p.rot, p.theta
    if p.scaling == lg.LG_ROPE_BASE:
        theta = theta * p.factor ** (rot / (rot - 2))
    out = []
    if p.scaling == lg.LG_ROPE_YARN:
        def pair(turns):
            return rot * math.log(p.orig_len / (turns * 2 * math.pi)) / (2 * math.log(theta))
        a = max(math.floor(pair(p.beta_fast)), 0)
        b = max(min(math.ceil(pair(p.beta_slow)), rot - 1) - a, 0.001)
    for i in range(rot // 2):
        f = theta ** (-2 * i / rot)
        w = 1.0
        if p.scaling == lg.LG_ROPE_LINEAR:
            w = 0.0
        elif p.scaling == lg.LG_ROPE_BANDS:
            w = min(max((p.orig_len * f / (2 * math.pi) - p.low) / (p.high - p.low), 0.0), 1.0)
        elif p.scaling == lg.LG_ROPE_YARN:
            w = 1.0 - min(max((i - a) / b, 0.0), 1.0)
        out.append(f * (w + (1 - w) / p.factor))
    return np.array(out)


def rotate(x, pos, p):
    """x [T][H][d] (numpy fp64) at positions pos [T]"""
    ang = np.asarray(pos, dtype=np.float64)[:, None] * frequencies(p, x.shape[-1])[None]
    c, s = np.cos(ang)[:, None] * p.mscale, np.sin(ang)[:, None] * p.mscale
    y = x.copy()
    if p.layout == lg.LG_ROPE_HALF:
        a, b = x[..., :p.rot // 2], x[..., p.rot // 2:p.rot]
        y[..., :p.rot // 2], y[..., p.rot // 2:p.rot] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., 0:p.rot:2], x[..., 1:p.rot:2]
        y[..., 0:p.rot:2], y[..., 1:p.rot:2] = a * c - b * s, a * s + b * c
    return y


def pick(logits, seen, counts, penalty, bias, allowed):
    """(token, pmax, processed logits) of one row; logits fp32 values, everything in fp32 steps"""
    f = np.float32
    x = logits.astype(f).copy()
    V = len(x)
    if seen is not None:
        rep, pres, freq = (f(v) for v in penalty[:3])
        for t in np.nonzero(seen)[0]:
            x[t] = x[t] / rep if x[t] > 0 else x[t] * rep
            if counts[t] > 0:
                x[t] = (x[t] - freq * f(counts[t])) - pres
    for t, v in bias or []:
        if 0 <= t < V:
            x[t] = x[t] + f(v)
    if allowed is not None:
        x[~allowed] = -np.inf
    x[np.isnan(x)] = -np.inf
    m = x.max()
    if m == -np.inf:
        return -1, 0.0, x
    if m == np.inf:
        return int(np.argmax(x)), 1.0 / np.count_nonzero(x == m), x
    return int(np.argmax(x)), 1.0 / np.exp(x.astype(np.float64) - m).sum(), x


def pack(flags):
    """truth values [V] -> int32 words"""
    V = len(flags)
    b = np.zeros((V + 31) // 32 * 32, dtype=np.uint64)
    b[:V] = flags
    w = (b.reshape(-1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return w.view(np.int32)
