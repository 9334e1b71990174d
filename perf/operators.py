"""The operators around one model step of the guarded cache, as measurable cases.

A case names a `kind` and its sizes:

  attend  attention of a chunk of new tokens over the cache (lg_chunk_attend): query j of a sequence
          that added m rows sits at row r = len - m + j and sees the rows i <= r; with a window, only
          those with i > r - window or i < n_sink.  m = 1 is the decode step
  rope    rotary positions of a chunk's queries and keys, its keys and values joining the cache with
          the guard layer's sketches (lg_rope_append)
  pick    penalties for repeated tokens, biases and a grammar mask on the logits, the token they
          leave on top and its probability, which the token-level monitor reads (lg_pick_token)

The plain forms compute in 32 bits (the angles in 64) with elementary torch operations and round
once at the end.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # a decode step's layer of the 1.7B-class model at one sequence: latency is all of it
        dict(name="attend_one", kind="attend", H_q=16, H_kv=8, d=128, dtype="bf16", batch=1, new=1,
             n=1025, ragged=False, window=0, sink=0),
        # continuous batching with a sliding window and four sinks: 64 sequences of log-uniform
        # lengths, one token each
        dict(name="attend_window_b64", kind="attend", H_q=32, H_kv=8, d=128, dtype="bf16",
             batch=64, new=1, n=16381, ragged=True, window=4096, sink=4),
        # a few proposed tokens a sequence to be checked in one pass
        dict(name="attend_verify_b16", kind="attend", H_q=32, H_kv=8, d=128, dtype="bf16",
             batch=16, new=7, n=4099, ragged=True, window=0, sink=0),
        # chunked prefill of eight long requests, 8B-class heads
        dict(name="attend_chunk_b8", kind="attend", H_q=32, H_kv=8, d=128, dtype="bf16", batch=8,
             new=512, n=8192, ragged=False, window=0, sink=0),
        # two whole prompts: the largest case
        dict(name="attend_prompt_b2", kind="attend", H_q=32, H_kv=8, d=128, dtype="bf16", batch=2,
             new=12288, n=12288, ragged=False, window=0, sink=0),
        # ragged prompts under a window, small heads, 7 query heads to a kv-head
        dict(name="attend_prompt_window_d64", kind="attend", H_q=14, H_kv=2, d=64, dtype="bf16",
             batch=3, new=9001, n=9001, ragged=True, window=1024, sink=4),
        # a caller that keeps its cache in fp32, ragged chunks of odd sizes
        dict(name="attend_f32_b4", kind="attend", H_q=24, H_kv=8, d=128, dtype="f32", batch=4,
             new=301, n=2501, ragged=True, window=0, sink=0),
        # one token of one sequence joins the cache
        dict(name="rope_one", kind="rope", H_q=16, H_kv=8, d=128, dtype="bf16", batch=1, new=1,
             n=1025, ragged=False, layout="half", rot=128, scaling="plain", factor=1.0,
             theta=1e6, packed=True),
        # eight prompts of 4096 tokens, frequencies smoothed by wavelength for long contexts
        dict(name="rope_prompt_b8", kind="rope", H_q=32, H_kv=8, d=128, dtype="bf16", batch=8,
             new=4096, n=4096, ragged=False, layout="half", rot=128, scaling="bands", factor=8.0,
             theta=5e5, packed=True),
        # fp32, interleaved pairs on half of the head, chunks at far positions
        dict(name="rope_f32_far", kind="rope", H_q=12, H_kv=4, d=64, dtype="f32", batch=5, new=777,
             n=1999, ragged=True, layout="interleaved", rot=32, scaling="yarn", factor=16.0,
             theta=1e4, packed=False),
        # the token of one sequence from fp32 logits
        dict(name="pick_one", kind="pick", batch=1, V=151936, dtype="f32", hist=2500, grammar=False,
             bias=0, keep=False),
        # a batch under grammar masks and biases that keeps its processed logits; an odd vocabulary,
        # so rows start at every alignment
        dict(name="pick_b192", kind="pick", batch=192, V=128257, dtype="bf16", hist=4096,
             grammar=True, bias=40, keep=True),
    ]


MAX_FLOPS = 3 * 10 ** 12  # of a drawn attention (the largest listed case has 4.9e12)


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "rope", "pick"])
    if kind == "pick":
        V = _logint(rng, 8000, 200000)
        dtype = rng.choice(["bf16", "f32"])
        return dict(kind=kind, batch=min(_logint(rng, 1, 256), (50 << 20) // V), V=V, dtype=dtype,
                    hist=_logint(rng, 16, 16384), grammar=rng.random() < 0.5,
                    bias=rng.choice([0, 1, 17, 300]), keep=rng.random() < 0.5)
    H_kv = rng.choice([2, 4, 8])
    d = rng.choice([64, 128, 128])
    c = dict(kind=kind, H_q=H_kv * rng.randint(1, 8), H_kv=H_kv, d=d,
             dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), batch=_logint(rng, 1, 64),
             new=1 if rng.random() < 0.35 else _logint(rng, 2, 8192),
             n=_logint(rng, 2, 65536), ragged=rng.random() < 0.6)
    c["new"] = min(c["new"], c["n"])
    if kind == "rope":
        c.update(layout=rng.choice(["half", "half", "interleaved"]),
                 rot=rng.choice([16, d // 4, d // 2, d, d]), theta=rng.choice([1e4, 5e5, 1e6]),
                 scaling=rng.choice(["plain", "linear", "base", "bands", "yarn"]),
                 factor=rng.choice([2.0, 4.0, 8.0]), packed=rng.random() < 0.5)
    else:
        win = rng.random() < 0.5
        c.update(window=_logint(rng, 1, 8192) if win else 0,
                 sink=rng.choice([0, 1, 4, 64]) if win else 0)
    # padded sizes under a limit: scores of 2^32 elements, rows of 2 GB
    while True:
        rows = c["batch"] * c["n"] * H_kv * d * 4
        tok = c["batch"] * c["new"] * c["H_q"] * d * 4
        scores = c["batch"] * c["H_q"] * c["new"] * c["n"]
        flops = 4 * d * scores * (4 if c["dtype"] == "f32" else 1)
        if rows <= (2 << 30) and tok <= (1 << 30) and (
                kind == "rope" or (scores <= (1 << 32) and flops <= MAX_FLOPS)):
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


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(g, shape, case):
    return torch.randn(shape, generator=g, device=DEV, dtype=_dtype(case))


def _offsets(ms):
    off = [0]
    for m in ms:
        off.append(off[-1] + m)
    return off


def _cache_inputs(case, g):
    """K, V [1][H_kv][S][d] with a scale per kv-head, and where each sequence lies"""
    ns, ms = _sizes(case)
    cap = [n + 1 for n in ns]
    kv = []
    for _ in range(2):
        x = _normal(g, (1, case["H_kv"], sum(cap), case["d"]), case)
        x *= torch.rand((1, case["H_kv"], 1, 1), generator=g, device=DEV).mul_(1.5).add_(0.5).to(x.dtype)
        kv.append(x)
    return ns, ms, cap, _offsets(cap)[:-1], _offsets(ms), kv[0], kv[1]


def _prepare_cache(s, case, g):
    s.ns, s.ms, s.cap, seq_off, off, s.k, s.v = _cache_inputs(case, g)
    s.T, s.max_new, s.max_len = off[-1], max(s.ms), max(s.ns)
    s.seq_off = torch.tensor(seq_off, dtype=torch.int64, device=DEV)
    s.len = torch.tensor(s.ns, dtype=torch.int32, device=DEV)
    s.off = torch.tensor(off, dtype=torch.int32, device=DEV)
    if own:
        from paper_2604_10044_gb300 import lg
        s.cache = lg.Cache(1, case["H_kv"], case["d"], case["dtype"], seq_off, s.cap, s.ns, DEV,
                           "loopguard", s.k, s.v)
        s.sketch = s.cache.sketch
        s.chunk = lg.Chunk(s.off, s.T, s.max_new)
        s.p = lg.lg_default_params()
    else:
        s.sketch = torch.zeros((s.k.shape[2], case["H_kv"] * case["d"] // 32), dtype=torch.int32,
                               device=DEV)


def _attend_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = _State()
    _prepare_cache(s, case, g)
    s.q = _normal(g, (s.T, case["H_q"], case["d"]), case)
    return s


def _rope_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = _State()
    _prepare_cache(s, case, g)
    H_q, H_kv, d = case["H_q"], case["H_kv"], case["d"]
    if case["packed"]:  # one projection's output, [T][H_q + 2 H_kv][d]
        x = _normal(g, (s.T, H_q + 2 * H_kv, d), case)
        s.q, s.kn, s.vn = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    else:
        s.q, s.kn, s.vn = (_normal(g, (s.T, h, d), case) for h in (H_q, H_kv, H_kv))
    # consecutive positions, each sequence's last one anywhere up to 10^6 (rows pruned since)
    last = torch.randint(max(s.ns), 1000000, (case["batch"],), generator=g, device=DEV)
    t = torch.arange(s.T, device=DEV)
    b = torch.searchsorted(s.off[1:].long(), t, right=True)
    s.pos = (last[b] - (s.off.long()[b + 1] - 1 - t)).int()
    return s


def _pick_inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = _State()
    B, V, n = case["batch"], case["V"], case["hist"]
    nw = (V + 31) // 32
    # a healthy row spreads its mass; every other row is sure of a token it has produced before
    x = torch.randn((B, V), generator=g, device=DEV) * 2.0
    ids = (torch.rand((B, n), generator=g, device=DEV) ** 6 * V).long().clamp_(max=V - 1)
    sure = torch.arange(0, B, 2, device=DEV)
    x[sure, ids[sure, n - 1]] += 22.0
    s.logits = x.to(_dtype(case))
    gen = n // 2  # the first half is the prompt
    s.counts = torch.zeros((B, V), dtype=torch.int32, device=DEV)
    s.counts.scatter_add_(1, ids[:, gen:], torch.ones_like(ids[:, gen:], dtype=torch.int32))
    flag = torch.zeros((B, nw * 32), dtype=torch.bool, device=DEV)
    flag.scatter_(1, ids, True)
    s.seen = _pack(flag)
    s.penalty = torch.rand((B, 4), generator=g, device=DEV)
    s.penalty[:, 0] = 1.0 + 0.3 * s.penalty[:, 0]
    s.allowed = None
    if case["grammar"]:  # rows 4k leave a few tokens, rows 4k+1 most, the others all
        u = torch.rand((B, nw * 32), generator=g, device=DEV)
        lim = torch.tensor([0.001, 0.9, 2.0, 2.0], device=DEV)[torch.arange(B, device=DEV) % 4]
        s.allowed = _pack(u < lim[:, None])
    s.bias = None
    if case["bias"]:
        m = case["bias"]
        first = torch.randint(0, V, (B, 1), generator=g, device=DEV)
        ids = (first + torch.arange(m, device=DEV) * (V // m)) % V   # no token twice in a row
        s.bias = (torch.arange(0, B * m + 1, m, dtype=torch.int32, device=DEV),
                  ids.int().reshape(-1).contiguous(),
                  torch.randn(B * m, generator=g, device=DEV) * 3.0)
    s.tokens = torch.zeros(B, dtype=torch.int32, device=DEV)
    s.pmax = torch.zeros(B, dtype=torch.float32, device=DEV)
    s.kept = torch.empty_like(s.logits) if case["keep"] else None
    return s


def _pack(flag):
    """[B][32 w] truth values -> [B][w] words, column 32 w + j in bit j"""
    B = flag.shape[0]
    bit = torch.ones(32, dtype=torch.int64, device=DEV) << torch.arange(32, device=DEV)
    word = (flag.view(B, -1, 32) * bit).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int()


def _unpack(words, V):
    bit = torch.arange(32, device=DEV)
    return ((words[:, :, None] >> bit) & 1).bool().view(words.shape[0], -1)[:, :V]


def _rope_params(case):
    from paper_2604_10044_gb300 import lg
    kind = dict(plain=lg.LG_ROPE_PLAIN, linear=lg.LG_ROPE_LINEAR, base=lg.LG_ROPE_BASE,
                bands=lg.LG_ROPE_BANDS, yarn=lg.LG_ROPE_YARN)[case["scaling"]]
    return lg.lg_default_rope_params(
        case["d"], layout=lg.LG_ROPE_HALF if case["layout"] == "half" else lg.LG_ROPE_INTERLEAVED,
        rot=case["rot"], theta=case["theta"], scaling=kind, factor=case["factor"],
        orig_len=ORIG_LEN, **(dict(mscale=_mscale(case)) if case["scaling"] == "yarn" else {}))


def prepare(case, seed):
    kind = case["kind"]
    if kind == "attend":
        s = _attend_inputs(case, seed)
        s.out = torch.empty_like(s.q)
    elif kind == "rope":
        s = _rope_inputs(case, seed)
        s.out = torch.empty((s.T, case["H_q"], case["d"]), dtype=s.q.dtype, device=DEV)
    else:
        s = _pick_inputs(case, seed)
    s.case = case
    if own:
        from paper_2604_10044_gb300 import lg
        if kind == "attend":
            n = lg.lg_chunk_workspace_size(s.cache, s.chunk, case["H_q"], s.max_len)
            s.ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        elif kind == "rope":
            s.rope = _rope_params(case)
        else:
            s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s.case
    kind = case["kind"]
    if own:
        from paper_2604_10044_gb300 import lg
        if kind == "attend":
            lg.lg_chunk_attend(s.cache, s.chunk, 0, s.q, case["H_q"], case["d"] ** -0.5,
                               case["window"], case["sink"], s.out, s.max_len, s.ws)
            return s.out
        if kind == "rope":
            lg.lg_rope_append(s.cache, s.chunk, 0, s.q, s.kn, s.vn, s.pos, s.rope, s.out, s.p)
            return dict(q=s.out, k=s.k, v=s.v, sketch=s.sketch)
        lg.lg_pick_token(s.logits, s.seen, s.counts, s.penalty, s.bias, s.allowed, s.tokens,
                         s.pmax, s.status, s.kept)
        return dict(token=s.tokens, pmax=s.pmax, logits=s.kept)
    return dict(attend=_plain_attend, rope=_plain_rope, pick=_plain_pick)[kind](s)


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
    K, V = s.k[0][:, rows].float(), s.v[0][:, rows].float()                       # [H_kv][B][n][d]
    Q = s.q[toks].float().view(B, s.max_new, H_kv, g, d).permute(2, 0, 3, 1, 4)
    Q = Q.reshape(H_kv, B, g * s.max_new, d)
    S = (Q @ K.transpose(2, 3)).mul_(d ** -0.5).view(H_kv, B, g, s.max_new, s.max_len)
    r = (n - new)[:, None] + j[None]                                              # [B][m]
    hidden = i > r[..., None]
    if case["window"]:
        hidden |= (i <= r[..., None] - case["window"]) & (i >= case["sink"])
    S.masked_fill_(hidden[None, :, None], -math.inf)
    S.sub_(S.amax(-1, keepdim=True)).exp_()
    tot = S.sum(-1, keepdim=True)
    O = (S.view(H_kv, B, g * s.max_new, s.max_len) @ V).view(H_kv, B, g, s.max_new, d) / tot
    t = torch.arange(s.T, device=DEV)
    b = torch.searchsorted(off[1:], t, right=True)
    O = O.permute(1, 3, 0, 2, 4)[b, t - off[b]]                                   # [T][H_kv][g][d]
    s.out.copy_(O.reshape(s.T, case["H_q"], d))
    return s.out


ORIG_LEN = 8192  # the context that the frequencies were trained on
LOW, HIGH = 1.0, 4.0  # "bands": wavelengths over ORIG_LEN / LOW are stretched, under / HIGH kept
FAST, SLOW = 32.0, 1.0  # "yarn": turns over ORIG_LEN above which a frequency is kept, below stretched


def _mscale(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "yarn" else 1.0


def _frequencies(case):
    """radians a position of each pair, 64 bits"""
    rot, theta, factor = case["rot"], case["theta"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    if case["scaling"] == "base":
        theta = theta * factor ** (rot / (rot - 2.0))
    f = theta ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "bands":
        mix = ((ORIG_LEN * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        f = mix * f + (1 - mix) * f / factor
    elif case["scaling"] == "yarn":
        # the pair index at which a frequency makes so many turns over ORIG_LEN, rounded outwards
        def at(turns):
            return rot * math.log(ORIG_LEN / (turns * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(math.floor(at(FAST)), 0), min(math.ceil(at(SLOW)), rot - 1)
        mix = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        f = mix * f + (1 - mix) * f / factor
    return f


def _plain_rope(s):
    case = s.case
    rot, half = case["rot"], case["rot"] // 2
    angle = s.pos.double()[:, None] * _frequencies(case)
    c = (angle.cos() * _mscale(case)).float()[:, None]
    sn = (angle.sin() * _mscale(case)).float()[:, None]

    def turned(x):
        y = x.float()
        if case["layout"] == "half":
            a, b = y[..., :half], y[..., half:rot]
            z = torch.cat([a * c - b * sn, a * sn + b * c], -1)
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            z = torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)
        return torch.cat([z, y[..., rot:]], -1).to(x.dtype)

    s.out.copy_(turned(s.q))
    t = torch.arange(s.T, device=DEV)
    off = s.off.long()
    b = torch.searchsorted(off[1:], t, right=True)
    row = s.seq_off[b] + s.len.long()[b] - off[b + 1] + t
    s.k[0].index_copy_(1, row, turned(s.kn).transpose(0, 1))
    s.v[0].index_copy_(1, row, s.vn.transpose(0, 1))
    s.sketch.index_copy_(0, row, _pack(torch.signbit(s.vn).reshape(s.T, -1)))
    return dict(q=s.out, k=s.k, v=s.v, sketch=s.sketch)


def _plain_pick(s):
    B, V = s.logits.shape
    x = s.logits.float()
    rep, pres, freq = s.penalty[:, 0:1], s.penalty[:, 1:2], s.penalty[:, 2:3]
    x = torch.where(_unpack(s.seen, V), torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(s.counts > 0, (x - freq * s.counts.float()) - pres, x)
    if s.bias is not None:
        off, ids, val = s.bias
        e = torch.arange(ids.shape[0], device=DEV)
        b = torch.searchsorted(off[1:].long(), e, right=True)
        x.index_put_((b, ids.long()), val, accumulate=True)
    if s.allowed is not None:
        x.masked_fill_(~_unpack(s.allowed, V), -math.inf)
    m = x.amax(-1, keepdim=True)
    first = torch.where(x == m, torch.arange(V, device=DEV), V).amin(-1)
    none = m[:, 0] == -math.inf
    s.tokens.copy_(first.masked_fill(none, -1))
    s.pmax.copy_((1.0 / (x - m).exp().sum(-1)).masked_fill(none, 0.0))
    if s.kept is not None:
        s.kept.copy_(x)
    return dict(token=s.tokens, pmax=s.pmax, logits=s.kept)


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
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "pick":
        B, V = case["batch"], case["V"]
        return dict(bytes=B * (V * es * (2 if case["keep"] else 1) +
                               V // 8 * (2 if case["grammar"] else 1) + 8 * case["bias"] + 24),
                    flops=0)
    ns, ms = _sizes(case)
    H_q, H_kv, d = case["H_q"], case["H_kv"], case["d"]
    if case["kind"] == "rope":
        T = sum(ms)
        return dict(bytes=T * (2 * (H_q + 2 * H_kv) * d * es + H_kv * d // 8 + 4),
                    flops=T * (H_q + H_kv) * case["rot"] * 3)
    pairs = rows = 0
    for n, m in zip(ns, ms):
        p, r = _pairs(n, m, case["window"], case["sink"])
        pairs, rows = pairs + p, rows + r
    return dict(bytes=2 * rows * H_kv * d * es + 2 * sum(ms) * H_q * d * es,
                flops=4 * d * H_q * pairs)


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    return dict(attend=_exact_attend, rope=_exact_rope, pick=_exact_pick)[case["kind"]](case, seed)


def _exact_attend(case, seed):
    s = _attend_inputs(case, seed)
    H_q, H_kv, d = case["H_q"], case["H_kv"], case["d"]
    out = torch.zeros((s.T, H_q, d), dtype=torch.float64, device=DEV)
    if sum(n * m for n, m in zip(s.ns, s.ms)) * H_q * d > 2 * 10 ** 12:
        return None
    o = t = 0
    for n, m, cap in zip(s.ns, s.ms, s.cap):
        for h in range(H_q):
            K, V = (x[0, h // (H_q // H_kv), o:o + n].double() for x in (s.k, s.v))
            for a in range(0, m, 4096):
                e = min(m, a + 4096)
                z = s.q[t + a:t + e, h].double() @ K.T / math.sqrt(d)
                dist = torch.arange(n - m + a, n - m + e, device=DEV)[:, None] - torch.arange(n, device=DEV)
                see = dist >= 0
                if case["window"]:
                    see &= (dist < case["window"]) | (torch.arange(n, device=DEV) < case["sink"])
                z = torch.where(see, z, torch.full_like(z, -math.inf))
                w = torch.exp(z - z.max(-1, keepdim=True).values)
                out[t + a:t + e, h] = w @ V / w.sum(-1, keepdim=True)
        o, t = o + cap, t + m
    return out


def _exact_rope(case, seed):
    s = _rope_inputs(case, seed)
    rot = case["rot"]
    turn = torch.polar(torch.full((), _mscale(case), dtype=torch.float64, device=DEV),
                       s.pos.double()[:, None] * _frequencies(case))[:, None]

    def turned(x):
        y = x.double().clone()
        if case["layout"] == "half":
            z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * turn
            y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
        else:
            z = torch.complex(y[..., 0:rot:2].contiguous(), y[..., 1:rot:2].contiguous()) * turn
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        return y

    K, kn = s.k.double(), turned(s.kn)
    o = t = 0
    for n, m, cap in zip(s.ns, s.ms, s.cap):
        K[0, :, o + n - m:o + n] = kn[t:t + m].transpose(0, 1)
        o, t = o + cap, t + m
    return dict(q=turned(s.q), k=K, v=None, sketch=None)


def _exact_pick(case, seed):
    s = _pick_inputs(case, seed)
    B, V = s.logits.shape
    x = s.logits.double()
    p = s.penalty.double()
    for b in range(B):
        word = torch.arange(V, device=DEV) // 32
        bit = torch.arange(V, device=DEV) % 32
        hit = ((s.seen[b, word] >> bit) & 1).bool()
        x[b] = torch.where(hit, torch.where(x[b] > 0, x[b] / p[b, 0], x[b] * p[b, 0]), x[b])
        x[b] -= torch.where(s.counts[b] > 0, p[b, 1] + p[b, 2] * s.counts[b], torch.zeros_like(x[b]))
        if s.bias is not None:
            lo, hi = case["bias"] * b, case["bias"] * (b + 1)
            x[b, s.bias[1][lo:hi].long()] += s.bias[2][lo:hi].double()
        if s.allowed is not None:
            x[b, ~((s.allowed[b, word] >> bit) & 1).bool()] = -math.inf
    pm = torch.softmax(x, -1).amax(-1)
    return dict(token=None, pmax=torch.nan_to_num(pm, nan=0.0),
                logits=x if case["keep"] else None)
