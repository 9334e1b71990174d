"""Plain 64-bit forms of a 4-bit cache's rows, of attention over them, and of the verification of drafted
tokens.

Tolerances of the attention for few query rows (w the weights, s and lo a value's scale and least value,
c its code; a rounding to bf16 is off by 2^-8 at most):
  score   the products are exact; two matrix products of a group's sum and the groups' joining lose 2^-22
          of Z = scale sum_e s |q_e| 15; the sum of q times lo enters in two bf16 terms, off by 2^-16 of
          scale sum_groups |lo| |sum q|:  z_err is the sum of both
  result  a weight rounded to bf16 and again with the scale: 2 2^-8 of w s |c - 8|; the weights of lo + 8 s
          rounded once, alike for both: 2^-8 of w |lo + 8 s|; sums over at most 64 products of a warp lose
          64 2^-23 = 2^-17 of what they sum, which is w |lo|, w s (8 of it at the end) and w s |c - 8|, each
          by itself, also where the three cancel; the result's own rounding 2^-8; every weight and the
          normaliser off by z_err + 2^-20 each:
          |d| <= 2^-8 |ref| + 2^-7 sum w s |c - 8| + 2^-8 sum w |lo + 8 s|
                 + 2^-17 sum w (s |c - 8| + |lo| + 8 s) + 2 (z_err + 2^-20) sum w |v|
For many query rows the values are rounded to bf16 (2^-8 of each key element in a score: z_err grows by
2^-8 scale sum |q| |k|; 2^-8 of each value) and then go the way of a bf16 cache, whose weights are rounded
once.
"""
import math

import numpy as np
import torch

from paper_2604_10044_gb300 import lg

SHIFT = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28])


def quantised(x):
    """(codes, scale, least) of heads [..., d] of bf16, 4 groups each; a poisoned group has scale NaN"""
    g = x.float().unflatten(-1, (4, x.shape[-1] // 4))
    fine = torch.isfinite(g).all(-1)
    lo = g.amin(-1)
    rng = g.amax(-1) - lo
    fine &= rng < 2.0 ** 118
    s = (rng * np.float32(1 / 15)).bfloat16().float()
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    d = (g - lo[..., None]).double()                      # the subtraction in fp32
    sd = s.double()[..., None]
    c = torch.where(sd > 0, d / torch.where(sd > 0, sd, 1.0), torch.zeros_like(d)).round().clamp(0, 15)
    c = torch.where(fine[..., None], c, torch.zeros_like(c))
    nan = torch.full_like(s, math.nan)
    return c.long(), torch.where(fine, s, nan), torch.where(fine, lo, torch.zeros_like(lo))


def packed(x):
    """rows of bytes [..., d/2 + 16] of heads [..., d]"""
    c, s, lo = quantised(x)
    w = (c.flatten(-2).unflatten(-1, (-1, 8)) << SHIFT).sum(-1)
    sb = torch.where(torch.isnan(s), torch.full_like(w[..., :4], 0x7fff),
                     s.bfloat16().view(torch.int16).long() & 0xffff)
    par = sb | (lo.bfloat16().view(torch.int16).long() & 0xffff) << 16
    word = torch.cat([w, par], -1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int().view(torch.uint8)


def parts(row):
    """(codes, scale, least), each [..., d] in 64 bits"""
    d = (row.shape[-1] - 16) * 2
    word = row.contiguous().view(torch.int32).long() & 0xffffffff
    c = (word[..., :d // 8, None] >> SHIFT & 15).flatten(-2).double()
    par = row[..., d // 2:].contiguous().view(torch.bfloat16).double()
    return (c, par[..., 0::2].repeat_interleave(d // 4, -1),
            par[..., 1::2].repeat_interleave(d // 4, -1))


def values(row):
    c, s, lo = parts(row)
    return c * s + lo


class Batch:
    """A 4-bit cache whose sequences hold ns[b] rows, ms[b] of them new, with queries; gaps of two slots
    between sequences.  Every byte outside the rows is 0xff (NaN parameters)."""

    def __init__(self, ns, ms, H_kv=2, g=4, d=128, L=1, seed=0, device="cuda:0", spread=1.0,
                 pad_rows=3, layer=0):
        self.ns, self.ms, self.H_kv, self.g, self.d, self.L = ns, ms, H_kv, g, d, L
        self.H_q, self.device, self.layer = H_kv * g, device, layer
        gen = torch.Generator().manual_seed(seed)
        cap = np.array([n + 2 for n in ns], dtype=np.int32)
        self.seq = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int64)
        S = int(cap.sum())
        self.k = torch.full((L, H_kv, S, d // 2 + 16), 255, dtype=torch.uint8)
        self.v = self.k.clone()
        for o, n in zip(self.seq, ns):
            for x, a in ((self.k, spread), (self.v, 1.0)):
                y = torch.randn((L, H_kv, n, d), generator=gen) * a + 0.3
                x[:, :, o:o + n] = packed(y.bfloat16())
        self.T = sum(ms) + pad_rows
        self.q = torch.full((self.T, self.H_q, d), math.nan, dtype=torch.bfloat16)
        self.q[:sum(ms)] = torch.randn((sum(ms), self.H_q, d), generator=gen).bfloat16()
        self.cap = cap

    def to_device(self):
        dev = self.device
        self.cache = lg.Cache(self.L, self.H_kv, self.d, "q4", self.seq, self.cap,
                              np.array(self.ns, dtype=np.int32), dev, "loopguard", self.k.to(dev),
                              self.v.to(dev))
        ch = lg.Chunk.of(self.ms, dev)
        self.chunk = lg.Chunk(ch.off, self.T, ch.max_new)
        self.qd = self.q.to(dev)
        self.max_len = max(max(self.ns), 1)
        n = lg.lg_chunk_workspace_size(self.cache, self.chunk, self.H_q, self.max_len)
        assert n > 0 and n % 256 == 0
        self.ws = torch.full((n,), 0xff, dtype=torch.uint8, device=dev)
        return self

    def attend(self, window=0, sink=0, stream=None):
        """the call's output, rows it may not write still 7"""
        out = torch.full_like(self.qd, 7.0)
        lg.lg_chunk_attend(self.cache, self.chunk, self.layer, self.qd, self.H_q, self.d ** -0.5,
                           window, sink, out, self.max_len, self.ws, stream)
        return out

    def reference(self, window=0, sink=0, wide=False):
        """(ref, tol) of every query row"""
        ref = torch.full((self.T, self.H_q, self.d), 7.0, dtype=torch.float64)
        tol = torch.zeros_like(ref)
        t = 0
        for o, n, m in zip(self.seq, self.ns, self.ms):
            for h in range(self.H_q if m else 0):
                K = self.k[self.layer, h // self.g, o:o + n]
                V = self.v[self.layer, h // self.g, o:o + n]
                r, e, _ = attention(self.q[t:t + m, h], K, V, n, m, self.d ** -0.5, window, sink, wide)
                ref[t:t + m, h], tol[t:t + m, h] = r, e
            t += m
        return ref, tol


def attention(q, K, V, n, m, scale, window=0, sink=0, wide=False, suffix=0):
    """(result, tolerance, statistics) of queries [m][d] over rows of bytes; statistics and their
    tolerances [m][2][4] of {m, l, H, S}"""
    q = q.double()
    ck, sk, lk = parts(K)
    cv, sv, lv = parts(V)
    k, v = ck * sk + lk, cv * sv + lv
    i, r = torch.arange(n), torch.arange(n - m, n)[:, None]
    see = i <= r
    if window:
        see &= (i > r - window) | (i < sink)
    z = torch.where(see, q @ k.T * scale, -math.inf)
    # what the scores lose, the largest over the rows a query sees
    zb = scale * 15 * (q.abs() @ sk.T) * 2.0 ** -22
    d = q.shape[-1]
    sums = q.unflatten(-1, (4, d // 4)).sum(-1).abs().repeat_interleave(d // 4, -1) / (d // 4)
    zb += scale * (sums @ lk.abs().T) * 2.0 ** -16
    if wide:
        zb += scale * (q.abs() @ k.abs().T) * 2.0 ** -8
    zerr = torch.where(see, zb, 0.0).amax(-1, keepdim=True)
    w = torch.softmax(z, -1)
    ref = w @ v
    big = w @ v.abs()
    tol = 2.0 ** -8 * ref.abs() + 2 * (zerr + 2.0 ** -20) * big
    if wide:
        tol += 2 * 2.0 ** -8 * big + 2.0 ** -12 * big
    else:
        mid = (lv + 8 * sv).abs()
        tol += 2.0 ** -7 * (w @ (sv * (cv - 8).abs())) + 2.0 ** -8 * (w @ mid)
        tol += 2.0 ** -17 * (w @ (sv * (cv - 8).abs() + lv.abs() + 8 * sv))
    top = z.amax(-1)
    p = (z - top[:, None]).exp()
    l = p.sum(-1)
    lw = torch.where(see, torch.log_softmax(z, -1), 0.0)
    H = -(w * lw).sum(-1)
    S = w[:, max(0, n - suffix):].sum(-1) if suffix else torch.zeros(m)
    e = zerr[:, 0]
    rel = 2 * e + 2.0 ** -20 + n * 2.0 ** -24  # of a weight, and of a sum of them
    st = torch.stack([torch.stack([top, l, H, S], -1),
                      torch.stack([e + 2.0 ** -22 * top.abs(), rel * l,
                                   rel * (2 + (w * lw.abs()).sum(-1) + H), rel * (S + 2.0 ** -20)], -1)], 1)
    return ref, tol, st


def verify(x, ms, tokens, draft, temp, u, r):
    """(picked, accepted) as lg_verify_draft defines them, in 64 bits, a sequence at a time"""
    T, V = x.shape
    picked, accepted, t = [], [], 0
    for b, m in enumerate(ms):
        tau = 1.0 if temp is None else float(temp[b])

        def p_of(row):
            z = x[row].double().clone()
            z[torch.isnan(z)] = -math.inf
            top = z.max()
            p = torch.zeros(V, dtype=torch.float64)
            if top == -math.inf:
                return p
            if not tau > 2.0 ** -60:
                p[int(torch.nonzero(z == top)[0])] = 1.0
                return p
            if top == math.inf:
                e = (z == top).double()
            else:
                e = ((z - top) / min(tau, 2.0 ** 40)).exp()
                e[z == -math.inf] = 0.0
            return e / e.sum()

        def q_of(row):
            y = int(tokens[row + 1])
            q = torch.zeros(V, dtype=torch.float64)
            if not 0 <= y < V:
                return q
            if draft is None:
                q[y] = 1.0
                return q
            q = draft[row].double().clone()
            q[~(q > 0)] = 0.0
            return q

        a = 0
        while a < m - 1:
            y = int(tokens[t + a + 1])
            if not 0 <= y < V or not float(u[t + a]) * float(q_of(t + a)[y]) < float(p_of(t + a)[y]):
                break
            a += 1
        out = [-1] * m
        for j in range(min(a, m)):
            out[j] = int(tokens[t + j + 1])
        if m:
            p = p_of(t + a)
            w = (p - q_of(t + a)).clamp(min=0) if a < m - 1 else p
            if not (w * 2.0 ** 62).round().sum() > 0:
                w = p
            if w.sum() > 0:
                rr = float(r[b])
                rr = 0.0 if not rr > 0 else min(rr, 1 - 2.0 ** -60)
                cum = w.cumsum(0)
                over = torch.nonzero(cum > rr * cum[-1])
                if rr >= 1 - 2.0 ** -53 or not len(over):
                    out[a] = int(torch.nonzero(w > 0)[-1])
                else:
                    out[a] = int(over[0])
        picked += out
        accepted.append(a if m else 0)
        t += m
    return picked, accepted
