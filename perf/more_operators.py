"""The guarded cache in four bits and the drafted decode step over it, as measurable cases.

A case names a `kind` and its sizes:

  decode  attention of one new token a sequence over a 4-bit cache, with the statistics that the
          guard reads (lg_decode_attend)
  attend  attention of a chunk of new tokens over a 4-bit cache (lg_chunk_attend): query j of a
          sequence that added m rows sits at row r = len - m + j and sees the rows i <= r; with a
          window, only those with i > r - window or i < n_sink
  append  rotary positions of a chunk's queries and keys, its keys and values joining the 4-bit cache
          with the guard layer's sketches (lg_rope_append), and the rows read back as the values
          that they stand for (lg_read_rows)
  verify  drafted tokens against the target's probabilities, from given random numbers: how many
          stand, and the token that follows them (lg_verify_draft)

A head of d elements is held as four groups of d/4: codes c in 0..15, a scale s and a least value lo,
both bf16, and an element is lo + s c.  The plain forms compute in 32 bits with elementary torch
operations and round once at the end; angles, the borders between codes, and the sums of a
distribution that a random number is looked up in are in 64.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # a decode step's layer of the 1.7B-class model at one sequence: latency is all of it
        dict(name="decode_one", kind="decode", H_q=16, H_kv=8, d=128, batch=1, new=1, n=1025,
             ragged=False, window=0, sink=0),
        # continuous batching: 64 sequences of log-uniform lengths, 8B-class heads
        dict(name="decode_b64", kind="decode", H_q=32, H_kv=8, d=128, batch=64, new=1, n=16381,
             ragged=True, window=0, sink=0),
        # one far request, whose rows are divided over the whole GPU
        dict(name="decode_long", kind="decode", H_q=32, H_kv=8, d=128, batch=1, new=1, n=262143,
             ragged=False, window=0, sink=0),
        # a few drafted tokens a sequence to be checked in one pass
        dict(name="attend_verify_b16", kind="attend", H_q=32, H_kv=8, d=128, batch=16, new=5,
             n=16411, ragged=True, window=0, sink=0),
        # the same for small heads, 7 query heads to a kv-head, under a window with sinks
        dict(name="attend_verify_window_d64", kind="attend", H_q=14, H_kv=2, d=64, batch=48, new=4,
             n=9001, ragged=True, window=1024, sink=4),
        # chunked prefill of eight long requests: the largest case
        dict(name="attend_chunk_b8", kind="attend", H_q=32, H_kv=8, d=128, batch=8, new=512, n=8192,
             ragged=False, window=0, sink=0),
        # one token of one sequence joins the cache
        dict(name="append_one", kind="append", H_q=16, H_kv=8, d=128, batch=1, new=1, n=1025,
             ragged=False, theta=1e6),
        # ragged prompts of up to 4096 tokens
        dict(name="append_prompt_b8", kind="append", H_q=32, H_kv=8, d=128, batch=8, new=4096,
             n=4096, ragged=True, theta=5e5),
        # four drafts of one sequence, fp32 logits
        dict(name="verify_one", kind="verify", batch=1, drafts=4, V=151936, dtype="f32",
             certain=False, ragged=False),
        # a batch of up to six drafts each; an odd vocabulary, so rows start at every alignment
        dict(name="verify_b64", kind="verify", batch=64, drafts=6, V=128257, dtype="bf16",
             certain=False, ragged=True),
        # tokens drafted by looking up the prompt, which have no probabilities of their own
        dict(name="verify_lookup_b24", kind="verify", batch=24, drafts=9, V=32000, dtype="bf16",
             certain=True, ragged=True),
    ]


MAX_FLOPS = 5 * 10 ** 11  # of a drawn attention (the largest listed case has 5e11)


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "attend", "attend", "append", "verify", "verify"])
    if kind == "verify":
        V = _logint(rng, 2000, 200000)
        drafts = rng.randint(1, 9)
        return dict(kind=kind, batch=max(1, min(_logint(rng, 1, 128), (60 << 20) // (V * drafts))),
                    drafts=drafts, V=V, dtype=rng.choice(["bf16", "f32"]),
                    certain=rng.random() < 0.3, ragged=rng.random() < 0.6)
    H_kv = rng.choice([2, 4, 8])
    d = rng.choice([64, 128, 128])
    c = dict(kind=kind, H_q=H_kv * rng.randint(1, 8), H_kv=H_kv, d=d, batch=_logint(rng, 1, 64),
             new=1, n=_logint(rng, 2, 131072), ragged=rng.random() < 0.6)
    if kind != "decode":
        c["new"] = min(c["n"], _logint(rng, 1, 16) if rng.random() < 0.6 else _logint(rng, 17, 4096))
    if kind == "append":
        c["theta"] = rng.choice([1e4, 5e5, 1e6])
    else:
        win = kind == "attend" and rng.random() < 0.4
        c.update(window=_logint(rng, 1, 8192) if win else 0,
                 sink=rng.choice([0, 1, 4, 64]) if win else 0)
    # padded sizes under a limit: scores of 2^30 elements, rows of 4 GB in 32 bits
    while True:
        rows = c["batch"] * c["n"] * H_kv * d * 8
        tok = c["batch"] * c["new"] * c["H_q"] * d * 4
        scores = c["batch"] * c["H_q"] * c["new"] * c["n"]
        if rows <= (4 << 30) and tok <= (1 << 29) and (
                kind == "append" or (scores <= (1 << 30) and 4 * d * scores <= MAX_FLOPS)):
            return c
        if c["batch"] > 1:
            c["batch"] = (c["batch"] + 1) // 2
        elif c["new"] > 512:
            c["new"] = c["new"] // 2 + 1
        else:
            c["n"] = max(c["new"], c["n"] // 2)


# ------------------------------------------------------------------ inputs

class _State:
    pass


def _sizes(case):
    """(rows in use, new rows) of each sequence, the new ones counted in: all alike, or spread
    log-uniformly over [1/16, 1] of the largest"""
    b, n, m = case["batch"], case["n"], case["new"]
    if not case["ragged"]:
        return [n] * b, [m] * b
    ns, ms = [], []
    for i in range(b):
        u, w = (i * 0.6180339887498949 + 0.9999) % 1.0, (i * 0.7548776662466927 + 0.9999) % 1.0
        ms.append(max(1, int(m * 16.0 ** (w - 1.0) + 1e-9)))
        ns.append(max(ms[-1], int(n * 16.0 ** (u - 1.0) + 1e-9)))
    return ns, ms


def _drafts(case):
    """drafted tokens of each sequence: all alike, or from none to the most"""
    b, k = case["batch"], case["drafts"]
    if not case["ragged"]:
        return [k] * b
    return [int((k + 1) * ((i * 0.6180339887498949 + 0.9999) % 1.0)) for i in range(b)]


def _offsets(ms):
    off = [0]
    for m in ms:
        off.append(off[-1] + m)
    return off


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def _owner(off, T):
    """the sequence of each of T token rows"""
    return torch.searchsorted(off[1:].long(), torch.arange(T, device=DEV), right=True)


# A row of a head: d/8 words of eight codes, element 2i of a word in bits 4i and element 2i + 1 in
# bits 16 + 4i, i < 4; then four words of a group's scale (low half) and least value (high half), bf16.

def _quantised(x):
    """(codes, scale, least) of heads [..., d]: the scale is the range over 15 in bf16, a code the
    nearest integer to (x - least) / scale, ties to even, at most 15"""
    g = x.float().unflatten(-1, (4, x.shape[-1] // 4))
    lo = g.amin(-1).bfloat16()
    s = ((g.amax(-1) - lo.float()) / 15.0).bfloat16()
    d = (g - lo.float()[..., None]).double()
    c = torch.where(s[..., None] > 0, d / s.double()[..., None], torch.zeros_like(d))
    return c.round().clamp_(0, 15).int(), s, lo


def _packed(c, s, lo):
    """rows of bytes from codes [..., 4, d/4] and the groups' scales and least values [..., 4]"""
    w = c.flatten(-2).unflatten(-1, (-1, 8)).long()
    word = torch.zeros_like(w[..., 0])
    for e in range(8):
        word |= w[..., e] << (4 * (e // 2) + 16 * (e % 2))
    par = (s.view(torch.int16).long() & 0xffff) | (lo.view(torch.int16).long() & 0xffff) << 16
    word = torch.cat([word, par], -1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int().view(torch.uint8)


def _values(row, d):
    """the values that rows of bytes stand for, in 32 bits"""
    word = row.contiguous().view(torch.int32)
    shift = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=DEV, dtype=torch.int32)
    c = ((word[..., :d // 8, None] >> shift) & 15).flatten(-2).unflatten(-1, (4, d // 4))
    par = word[..., d // 8:].contiguous().view(torch.bfloat16).float().unflatten(-1, (4, 2))
    return (c * par[..., :1] + par[..., 1:]).flatten(-2)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV).bfloat16()


def _cache_inputs(s, case, g):
    """a cache of four bits of normal rows with a scale per kv-head, and where each sequence lies"""
    s.ns, s.ms = _sizes(case)
    H_kv, d = case["H_kv"], case["d"]
    s.cap = [n + 1 for n in s.ns]
    seq_off, off, S = _offsets(s.cap)[:-1], _offsets(s.ms), sum(s.cap)
    kv = []
    for _ in range(2):
        x = torch.empty((1, H_kv, S, d // 2 + 16), dtype=torch.uint8, device=DEV)
        for h in range(H_kv):
            a = torch.rand((), generator=g, device=DEV) * 1.5 + 0.5
            x[0, h] = _packed(*_quantised(torch.randn((S, d), generator=g, device=DEV) * a))
        kv.append(x)
    s.k, s.v = kv
    s.T, s.max_new, s.max_len = off[-1], max(s.ms), max(s.ns)
    s.seq_off, s.len, s.off = _ints(seq_off, torch.int64), _ints(s.ns), _ints(off)
    s.seq_off_host = seq_off
    s.sketch = torch.zeros((S, H_kv * d // 32), dtype=torch.int32, device=DEV)


def _attend_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = _State()
    _cache_inputs(s, case, g)
    s.q = _normal(g, s.T, case["H_q"], case["d"])
    return s


def _append_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = _State()
    _cache_inputs(s, case, g)
    H_q, H_kv = case["H_q"], case["H_kv"]
    x = _normal(g, s.T, H_q + 2 * H_kv, case["d"])  # one projection's output
    s.q, s.kn, s.vn = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    # consecutive positions, each sequence's last one anywhere up to 10^6 (rows pruned since)
    last = torch.randint(max(s.ns), 1000000, (case["batch"],), generator=g, device=DEV)
    b = _owner(s.off, s.T)
    s.pos = (last[b] - (s.off.long()[b + 1] - 1 - torch.arange(s.T, device=DEV))).int()
    return s


def _verify_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = _State()
    B, V = case["batch"], case["V"]
    s.ms = [k + 1 for k in _drafts(case)]
    off = _offsets(s.ms)
    s.T, s.max_new, s.off = off[-1], max(s.ms), _ints(off)
    # a target that is sure of a few tokens, and a draft model that sees nearly the same
    x = torch.randn((s.T, V), generator=g, device=DEV) * 2.0
    few = torch.randint(0, V, (s.T, 6), generator=g, device=DEV)
    x.scatter_add_(1, few, torch.rand((s.T, 6), generator=g, device=DEV) * 8.0 + 6.0)
    y = x + torch.randn((s.T, V), generator=g, device=DEV) * 0.5
    s.logits = x if case["dtype"] == "f32" else x.bfloat16()
    p = y.softmax(-1)
    # the drafted tokens come from the draft model's probabilities, the first token of a row's
    # sequence from the step before
    cum = p.double().cumsum(-1)
    at = torch.rand((s.T, 1), generator=g, device=DEV, dtype=torch.float64) * cum[:, -1:]
    drawn = torch.searchsorted(cum, at, right=True).clamp_(max=V - 1)[:, 0]
    s.tokens = torch.cat([drawn[-1:], drawn[:-1]]).int()
    s.draft = None if case["certain"] else p if case["dtype"] == "f32" else p.bfloat16()
    s.u = torch.rand(s.T, generator=g, device=DEV)
    s.r = torch.rand(B, generator=g, device=DEV)
    # every fourth sequence takes the top token, the others sample
    s.temp = torch.rand(B, generator=g, device=DEV) * 0.6 + 0.6
    s.temp[3::4] = 0.0
    return s


def prepare(case, seed):
    kind = case["kind"]
    if kind == "verify":
        s = _verify_inputs(case, seed)
        s.picked = torch.empty(s.T, dtype=torch.int32, device=DEV)
        s.accepted = torch.empty(case["batch"], dtype=torch.int32, device=DEV)
    elif kind == "append":
        s = _append_inputs(case, seed)
        s.out = torch.empty((s.T, case["H_q"], case["d"]), dtype=torch.bfloat16, device=DEV)
        s.rows = [torch.empty_like(x, memory_format=torch.contiguous_format) for x in (s.kn, s.vn)]
    else:
        s = _attend_inputs(case, seed)
        s.out = torch.empty_like(s.q)
        s.stats = torch.empty((1, case["batch"], case["H_q"], 4), device=DEV)
    s.case = case
    if own:
        from paper_2604_10044_gb300 import lg
        s.chunk = lg.Chunk(s.off, s.T, s.max_new)
        if kind == "verify":
            s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
            n = lg.lg_verify_workspace_size(s.logits, s.chunk)
        else:
            s.cache = lg.Cache(1, case["H_kv"], case["d"], "q4", s.seq_off_host, s.cap, s.ns, DEV,
                               "loopguard", s.k, s.v)
            s.cache.sketch = s.sketch = s.cache.sketch
            s.p = lg.lg_default_params()
            n = 256
            if kind == "decode":
                n = lg.lg_workspace_size(s.cache, case["H_q"], 1, s.max_len)
            elif kind == "attend":
                n = lg.lg_chunk_workspace_size(s.cache, s.chunk, case["H_q"], s.max_len)
            else:
                s.rope = lg.lg_default_rope_params(case["d"], theta=case["theta"])
        s.ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


SUFFIX = 64  # rows of the suffix-mass statistic


# ------------------------------------------------------------------ one pass

def run(s):
    case = s.case
    kind = case["kind"]
    if own:
        from paper_2604_10044_gb300 import lg
        if kind == "verify":
            lg.lg_verify_draft(s.logits, s.chunk, s.tokens, s.draft, s.temp, s.u, s.r, s.picked,
                               s.accepted, s.ws, s.status)
            return dict(picked=s.picked, accepted=s.accepted)
        if kind == "append":
            lg.lg_rope_append(s.cache, s.chunk, 0, s.q, s.kn, s.vn, s.pos, s.rope, s.out, s.p)
            lg.lg_read_rows(s.cache, s.chunk, 0, s.rows[0], s.rows[1])
            return dict(q=s.out, k=s.rows[0], v=s.rows[1], sketch=s.sketch)
        if kind == "decode":
            lg.lg_decode_attend(s.cache, 0, 1, s.q, case["H_q"], case["d"] ** -0.5, s.out, s.stats,
                                SUFFIX, 0, s.max_len, s.ws)
            return dict(out=s.out, stats=s.stats)
        lg.lg_chunk_attend(s.cache, s.chunk, 0, s.q, case["H_q"], case["d"] ** -0.5,
                           case["window"], case["sink"], s.out, s.max_len, s.ws)
        return dict(out=s.out)
    return dict(decode=_plain_attend, attend=_plain_attend, append=_plain_append,
                verify=_plain_verify)[kind](s)


def _plain_attend(s):
    case = s.case
    H_kv, d, B = case["H_kv"], case["d"], case["batch"]
    g = case["H_q"] // H_kv
    n, off = s.len.long(), s.off.long()
    new = off[1:] - off[:-1]
    i = torch.arange(s.max_len, device=DEV)
    j = torch.arange(s.max_new, device=DEV)
    rows = s.seq_off[:, None] + torch.minimum(i[None], n[:, None] - 1)            # [B][n]
    toks = off[:-1, None] + torch.minimum(j[None], new[:, None] - 1)              # [B][m]
    K = _values(s.k[0], d)[:, rows]                                               # [H_kv][B][n][d]
    Q = s.q[toks].float().view(B, s.max_new, H_kv, g, d).permute(2, 0, 3, 1, 4)
    Q = Q.reshape(H_kv, B, g * s.max_new, d)
    S = (Q @ K.transpose(2, 3)).mul_(d ** -0.5).view(H_kv, B, g, s.max_new, s.max_len)
    del K
    r = (n - new)[:, None] + j[None]                                              # [B][m]
    hidden = i > r[..., None]
    if case["window"]:
        hidden |= (i <= r[..., None] - case["window"]) & (i >= case["sink"])
    S.masked_fill_(hidden[None, :, None], -math.inf)
    top = S.amax(-1, keepdim=True)
    P = (S - top).exp_()
    tot = P.sum(-1, keepdim=True)
    V = _values(s.v[0], d)[:, rows]
    O = (P.view(H_kv, B, g * s.max_new, s.max_len) @ V).view(H_kv, B, g, s.max_new, d) / tot
    t = torch.arange(s.T, device=DEV)
    b = _owner(s.off, s.T)
    O = O.permute(1, 3, 0, 2, 4)[b, t - off[b]]                                   # [T][H_kv][g][d]
    s.out.copy_(O.reshape(s.T, case["H_q"], d))
    if case["kind"] == "attend":
        return dict(out=s.out)
    P = (P / tot)[..., 0, :]                                                      # [H_kv][B][g][n]
    H = -torch.where(P > 0, P * P.log(), 0.0).sum(-1)
    suffix = torch.where(i >= n[:, None, None] - SUFFIX, P, 0.0).sum(-1)
    st = torch.stack([top[..., 0, 0], tot[..., 0, 0], H, suffix], -1)             # [H_kv][B][g][4]
    s.stats.copy_(st.permute(1, 0, 2, 3).reshape(1, B, case["H_q"], 4))
    return dict(out=s.out, stats=s.stats)


def _angles(case, pos):
    i = torch.arange(case["d"] // 2, dtype=torch.float64, device=DEV)
    return pos.double()[:, None, None] * case["theta"] ** (-2.0 * i / case["d"])


def _plain_append(s):
    case = s.case
    half = case["d"] // 2
    angle = _angles(case, s.pos)
    c, sn = angle.cos().float(), angle.sin().float()

    def turned(x):
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat([a * c - b * sn, a * sn + b * c], -1)

    s.out.copy_(turned(s.q))
    b = _owner(s.off, s.T)
    slot = s.seq_off[b] + s.len.long()[b] - s.off.long()[b + 1] + torch.arange(s.T, device=DEV)
    kn = _packed(*_quantised(turned(s.kn).bfloat16()))
    vn = _packed(*_quantised(s.vn))
    s.k[0].index_copy_(1, slot, kn.transpose(0, 1))
    s.v[0].index_copy_(1, slot, vn.transpose(0, 1))
    neg = torch.signbit(s.vn).reshape(s.T, -1, 32)
    bit = torch.ones(32, dtype=torch.int64, device=DEV) << torch.arange(32, device=DEV)
    word = (neg * bit).sum(-1)
    s.sketch.index_copy_(0, slot, torch.where(word >= 1 << 31, word - (1 << 32), word).int())
    for out, x in zip(s.rows, (s.k, s.v)):
        out.copy_(_values(x[0][:, slot], case["d"]).transpose(0, 1))
    return dict(q=s.out, k=s.rows[0], v=s.rows[1], sketch=s.sketch)


def _plain_verify(s):
    T, V = s.logits.shape
    B, off = s.case["batch"], s.off.long()
    b = _owner(s.off, T)
    t = torch.arange(T, device=DEV)
    ids = torch.arange(V, device=DEV)
    x = s.logits.double()
    temp = s.temp.double()[b, None]
    d = x - x.amax(-1, keepdim=True)
    top = torch.where(d == 0, ids, V).amin(-1)
    e = torch.where(temp > 0, (d / torch.where(temp > 0, temp, 1.0)).exp(),
                    (ids == top[:, None]).double())
    p = e / e.sum(-1, keepdim=True)
    drafted = t < off[b + 1] - 1            # rows whose outcome a draft names
    y = torch.where(drafted, s.tokens.long().roll(-1), 0)
    q = (ids == y[:, None]).double() if s.draft is None else s.draft.double()
    q = torch.where(drafted[:, None], q, 0.0)
    at = (t, y)
    stands = drafted & (s.u.double() * q[at] < p[at])
    # the first row of each sequence that does not stand; its last row never does
    first = torch.full((B,), T, device=DEV).scatter_reduce(0, b, torch.where(stands, T, t), "amin")
    n = first - off[:-1]
    w = (p - q)[first].clamp_(min=0)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, p[first])
    cum = w.cumsum(-1)
    token = (cum <= s.r.double()[:, None] * cum[:, -1:]).sum(-1)
    s.accepted.copy_(n)
    s.picked.copy_(torch.where(t < first[b], y, torch.where(t == first[b], token[b], -1)))
    return dict(picked=s.picked, accepted=s.accepted)


# ------------------------------------------------------------------ what a pass cannot do without

def _pairs(n, m, window, sink):
    """(query, row) pairs a sequence of n rows computes for its last m, and the rows any of them
    sees"""
    if not window:
        return m * (n - m) + m * (m + 1) // 2, n
    pairs = 0
    for r in range(n - m, n):
        lo = max(0, r + 1 - window)
        pairs += r + 1 - lo + min(sink, lo)
    lo = max(0, n - m + 1 - window)
    return pairs, n - lo + min(sink, lo)


def work(case):
    if case["kind"] == "verify":  # every row of logits, one row of draft probabilities a sequence
        es, V, T = 2 if case["dtype"] == "bf16" else 4, case["V"], sum(_drafts(case)) + case["batch"]
        return dict(bytes=V * es * (T + (0 if case["certain"] else case["batch"])) + 12 * T,
                    flops=3 * T * V)
    ns, ms = _sizes(case)
    H_q, H_kv, d = case["H_q"], case["H_kv"], case["d"]
    row = d // 2 + 16
    if case["kind"] == "append":
        T = sum(ms)
        return dict(bytes=T * (4 * H_q * d + 8 * H_kv * d + 2 * H_kv * row + H_kv * d // 8 + 4),
                    flops=T * ((H_q + H_kv) * d * 3 + 2 * H_kv * d * 5))
    pairs = rows = 0
    for n, m in zip(ns, ms):
        p, r = _pairs(n, m, case["window"], case["sink"])
        pairs, rows = pairs + p, rows + r
    return dict(bytes=2 * rows * H_kv * row + 4 * sum(ms) * H_q * d +
                (16 * case["batch"] * H_q if case["kind"] == "decode" else 0),
                flops=4 * d * H_q * pairs)


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    if case["kind"] == "verify":  # its outputs are whole numbers
        return None
    return dict(decode=_exact_attend, attend=_exact_attend,
                append=_exact_append)[case["kind"]](case, seed)


def _held(row, d):
    """values of rows of bytes, in 64 bits, byte by byte"""
    c = torch.empty((row.shape[0], d), dtype=torch.float64, device=DEV)
    for e in range(8):
        byte = row[:, (2 * (e % 2) + e // 4):d // 2:4].double()  # of every word
        nib = torch.floor(byte / 16) if e // 2 % 2 else torch.remainder(byte, 16)
        c[:, e::8] = nib
    par = row[:, d // 2:].contiguous().view(torch.bfloat16).double()
    return c * par[:, 0::2].repeat_interleave(d // 4, 1) + par[:, 1::2].repeat_interleave(d // 4, 1)


def _exact_attend(case, seed):
    s = _attend_inputs(case, seed)
    H_q, H_kv, d = case["H_q"], case["H_kv"], case["d"]
    if sum(n * m for n, m in zip(s.ns, s.ms)) * H_q * d > 2 * 10 ** 12:
        return None
    out = torch.zeros((s.T, H_q, d), dtype=torch.float64, device=DEV)
    stats = torch.zeros((1, case["batch"], H_q, 4), dtype=torch.float64, device=DEV)
    o = t = 0
    for b, (n, m, cap) in enumerate(zip(s.ns, s.ms, s.cap)):
        for h in range(H_kv):
            K, V = _held(s.k[0, h, o:o + n], d), _held(s.v[0, h, o:o + n], d)
            dist = torch.arange(n - m, n, device=DEV)[:, None] - torch.arange(n, device=DEV)
            see = dist >= 0
            if case["window"]:
                see &= (dist < case["window"]) | (torch.arange(n, device=DEV) < case["sink"])
            for f in range(h * H_q // H_kv, (h + 1) * H_q // H_kv):
                z = s.q[t:t + m, f].double() @ K.T / math.sqrt(d)
                z = torch.where(see, z, torch.full_like(z, -math.inf))
                lw = torch.log_softmax(z, -1)
                w = lw.exp()
                out[t:t + m, f] = w @ V
                if case["kind"] == "decode":
                    stats[0, b, f, 0] = z.max()
                    stats[0, b, f, 1] = (z - z.max()).exp().sum()
                    stats[0, b, f, 2] = -(w * lw).sum()
                    stats[0, b, f, 3] = w[0, max(0, n - SUFFIX):].sum()
        o, t = o + cap, t + m
    return dict(out=out, stats=stats) if case["kind"] == "decode" else dict(out=out)


def _exact_append(case, seed):
    s = _append_inputs(case, seed)
    half = case["d"] // 2
    a = _angles(case, s.pos)
    turn = torch.polar(torch.ones_like(a), a)
    q = torch.view_as_real(torch.complex(s.q[..., :half].double(), s.q[..., half:].double()) * turn)
    # the rows are the nearest of what four bits can hold, which is no number in 64 bits
    return dict(q=torch.cat([q[..., 0], q[..., 1]], -1), k=None, v=None, sketch=None)
