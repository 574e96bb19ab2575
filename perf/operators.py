"""Plain forms and measured cases of the attention-side operators: the per-head norm with the position rotation, the append
to a paged FB4 cache, and attention over that cache.

Three operators, in the order a layer uses them:
  rotate   q, k [T][heads][D] bf16 -> RMS norm of every head, rotation by one or several position axes, bf16
  append   the same for q and k, then k and v quantized to FB4 blocks of 32 channels and written to slots of a paged cache
  attend   softmax(scale * q k^T) v of the new tokens of several sequences over their pages of that cache

FB4 (block of 32 channels): e = floor(log2(max |x|)), element scale 2^(e-3); the dialect (8 of the integers 0..15) is the one
with the smallest summed error, among those whose largest magnitude fits the block's maximum, of the bins of the 8 group
maxima; an element is the nearest magnitude of the dialect at its 0.5-wide bin.  codes uint8 [..][D/2], low nibble first,
nibble = sign << 3 | index; meta int16 [..][D/32], bits 0-7 = e + 124, bits 8-12 = dialect.
"""
import numpy as np
import torch

own = False

# the 32 dialects (the quantizer's built-in formatbook)
BOOK = (
    (0, 1, 2, 3, 4, 5, 6, 8), (0, 1, 2, 4, 5, 6, 7, 8), (0, 1, 2, 3, 4, 5, 7, 9), (0, 1, 2, 4, 6, 7, 8, 9),
    (0, 1, 2, 3, 4, 6, 8, 10), (0, 1, 2, 3, 5, 7, 9, 10), (0, 1, 2, 4, 6, 8, 9, 10), (0, 1, 2, 3, 4, 6, 8, 11),
    (0, 1, 2, 3, 5, 7, 9, 11), (0, 1, 2, 4, 6, 8, 10, 11), (0, 1, 2, 3, 4, 6, 8, 12), (0, 1, 2, 3, 5, 7, 9, 12),
    (0, 1, 2, 4, 6, 8, 10, 12), (0, 2, 4, 6, 8, 10, 11, 12), (0, 1, 2, 3, 4, 6, 9, 13), (0, 1, 2, 3, 5, 7, 10, 13),
    (0, 1, 2, 4, 6, 8, 10, 13), (0, 1, 2, 4, 6, 9, 11, 13), (0, 2, 4, 6, 8, 10, 12, 13), (0, 1, 2, 3, 4, 6, 9, 14),
    (0, 1, 2, 3, 5, 7, 10, 14), (0, 1, 2, 4, 6, 8, 11, 14), (0, 1, 2, 4, 6, 9, 12, 14), (0, 1, 3, 5, 7, 9, 12, 14),
    (0, 2, 4, 6, 8, 10, 12, 14), (0, 1, 2, 3, 4, 6, 9, 15), (0, 1, 2, 3, 5, 7, 10, 15), (0, 1, 2, 4, 6, 8, 11, 15),
    (0, 1, 2, 4, 6, 9, 12, 15), (0, 1, 3, 5, 7, 9, 12, 15), (0, 1, 3, 5, 7, 10, 13, 15), (0, 2, 4, 6, 8, 11, 13, 15),
)
EPS = 1e-6
DEV = "cuda"


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one new token of an autoregressive model: all latency
        dict(name="rotate one token", op="rotate", tokens=1, q_heads=32, k_heads=8, dim=128, axes=1, interleaved=False, height=0, width=0),
        # one latent frame of a video model (30 x 52 positions), three position axes, adjacent pairs
        dict(name="rotate a frame", op="rotate", tokens=1560, q_heads=12, k_heads=12, dim=128, axes=3, interleaved=True, height=30, width=52),
        # a whole clip of 21 such frames: the largest
        dict(name="rotate a clip", op="rotate", tokens=32760, q_heads=12, k_heads=12, dim=128, axes=3, interleaved=True, height=30, width=52),
        # one new token for each of 64 sequences
        dict(name="append 64 x 1", op="append", seqs=64, tokens=1, q_heads=32, kv_heads=8, dim=128, axes=1, interleaved=False, height=0, width=0, page=16),
        # ragged prompts of an odd length, narrow heads, padded rows at the end of the batch
        dict(name="append 3 x 1365", op="append", seqs=3, tokens=1365, q_heads=16, kv_heads=4, dim=64, axes=1, interleaved=False, height=0, width=0, page=32),
        # a clip's keys and values at once
        dict(name="append a clip", op="append", seqs=1, tokens=32760, q_heads=12, kv_heads=12, dim=128, axes=3, interleaved=True, height=30, width=52, page=64),
        # one token over a short cache: latency
        dict(name="attend 1 over 1023", op="attend", seqs=1, q_min=1, q_max=1, kv_min=1023, kv_max=1023, q_heads=8, kv_heads=8, dim=128, page=16, causal=True, window=0),
        # one token of one sequence over the longest cache
        dict(name="attend 1 over 75600", op="attend", seqs=1, q_min=1, q_max=1, kv_min=75600, kv_max=75600, q_heads=12, kv_heads=12, dim=128, page=64, causal=True, window=0),
        # a serving batch: 64 sequences of very different lengths, four query heads to a cache head
        dict(name="attend 64 x 1, ragged", op="attend", seqs=64, q_min=1, q_max=1, kv_min=131, kv_max=8191, q_heads=32, kv_heads=8, dim=128, page=16, causal=True, window=0),
        # drafted tokens checked together, with a sliding window; narrow heads
        dict(name="attend 8 x 6, window", op="attend", seqs=8, q_min=3, q_max=6, kv_min=2000, kv_max=20479, q_heads=16, kv_heads=4, dim=64, page=32, causal=True, window=4096),
        # prompts in chunks: causal against all that is cached
        dict(name="attend 4 x 1024, causal", op="attend", seqs=4, q_min=515, q_max=1024, kv_min=1024, kv_max=4096, q_heads=32, kv_heads=8, dim=128, page=16, causal=True, window=0),
        # a new frame over a cached clip, every token seeing all of it
        dict(name="attend a frame", op="attend", seqs=1, q_min=1560, q_max=1560, kv_min=32760, kv_max=32760, q_heads=12, kv_heads=12, dim=128, page=64, causal=False, window=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend"])
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16])
    group = rng.choice([1, 1, 2, 4, 7, 8])
    dim = rng.choice([64, 128, 128] if op == "attend" else [64, 96, 128, 128])
    if kv * group > 40:
        group = 1
    case = dict(op=op, q_heads=kv * group, dim=dim)
    if op != "attend":
        axes = rng.choice([1, 3])
        per_token = (kv * group + kv * (1 if op == "rotate" else 2)) * dim
        most = max(64, 32760 * (24 if op == "rotate" else 30) * 128 // per_token)
        seqs = 1 if op == "rotate" else _log(rng, 1, 64)
        tokens = _log(rng, 1, max(1, min(32760, most // seqs)))
        case |= dict(tokens=tokens, axes=axes, interleaved=rng.random() < 0.5, height=rng.randint(3, 48) if axes == 3 else 0,
                     width=rng.randint(3, 80) if axes == 3 else 0)
        case |= dict(k_heads=kv) if op == "rotate" else dict(kv_heads=kv, seqs=seqs, page=rng.choice([16, 32, 64, 128]))
        return case
    kind = rng.choice(["one", "few", "many"])
    seqs = _log(rng, 1, 96 if kind != "many" else 8)
    q_max = 1 if kind == "one" else _log(rng, 2, 24) if kind == "few" else _log(rng, 25, 2048)
    kv_max = min(75600, 75600 * 12 * 128 // (seqs * kv * dim), 500_000_000 // (seqs * q_max * kv * group))
    kv_max = _log(rng, 1, max(1, kv_max))
    kv_min = _log(rng, 1, kv_max)
    return case | dict(kv_heads=kv, seqs=seqs, q_min=rng.randint(1, q_max), q_max=q_max, kv_min=kv_min, kv_max=kv_max,
                       page=rng.choice([16, 32, 64, 128]), causal=rng.random() < 0.7, window=rng.choice([0, 0, 0, _log(rng, 1, 5000)]))


# ---------------------------------------------------------------------------------------------------- the format, plainly

_const = {}


def _tables():
    """qerr[bin][dialect] in quarter units, qvalue[dialect][bin], stage1[bin][dialect], book[dialect][index]"""
    if "t" not in _const:
        book = np.array(BOOK, np.int64)
        k = np.arange(32)
        index = ((book[:, None, 1:] + book[:, None, :-1]) <= k[None, :, None]).sum(2)             # [dialect][bin]
        err = np.abs(2 * k[None, :] + 1 - 4 * np.take_along_axis(book, index, 1))
        first = book[None, :, 7] == np.maximum(8, k[:, None] // 2)
        _const["t"] = [torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
                       for a in (err.T.astype(np.float32), index, first, book.astype(np.float32))]
    return _const["t"]


def _encode(x):
    """x float32 [..., D] -> (index with sign [..., D] uint8 0..15, dialect [..., D/32], scale byte [..., D/32])"""
    qerr, qvalue, stage1, _ = _tables()
    b = x.reshape(-1, 32)
    e = (torch.frexp(b.abs().amax(1)).exponent - 1).clamp(-124, 127)
    e = torch.where(b.abs().amax(1) == 0, torch.full_like(e, -124), e)
    bins = torch.floor(torch.ldexp(b.abs(), (4 - e)[:, None])).to(torch.int64).clamp_(max=31)
    groups = bins.view(-1, 8, 4).amax(2)
    err = qerr[groups].sum(1)
    key = torch.where(stage1[bins.amax(1)], err * 32 + torch.arange(32, device=x.device), float("inf"))
    did = key.amin(1).to(torch.int64) % 32
    idx = qvalue.view(-1)[did[:, None] * 32 + bins]
    code = (idx + 8 * torch.signbit(b).to(torch.int64)).to(torch.uint8)
    shape = (*x.shape[:-1], x.shape[-1] // 32)
    return code.view(x.shape), did.view(shape), (e + 124).view(shape)


def _values(code, did, scale):
    """what codes stand for, float32 (exact)"""
    book = _tables()[3]
    c = code.view(*did.shape, 32).to(torch.int64)
    m = book.view(-1)[did[..., None] * 8 + (c & 7)]
    v = torch.ldexp(torch.where(c >= 8, -m, m), (scale - 127)[..., None].to(torch.int32))
    return v.view(code.shape)


def _pack(code, did, scale):
    c = code.view(*code.shape[:-1], -1, 2)
    return (c[..., 0] | (c[..., 1] << 4)).contiguous(), (scale | (did << 8)).to(torch.int16)


def _unpack(codes, meta):
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    m = meta.to(torch.int64)
    return _values(code, (m >> 8) & 31, m & 255)


# ---------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _projection(g, tokens, width):
    """what a projection gives: a scale of its own for every token, heavy tails, a few outlier channels"""
    x = torch.randn(tokens, width, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(tokens, 1, generator=g, device=DEV))
    x *= 1 + 0.3 * torch.randn(tokens, width, generator=g, device=DEV).square_()
    out = torch.rand(width, generator=g, device=DEV) < 0.005
    return torch.where(out, x * 20, x).to(torch.bfloat16)


def _rope(case, pos0):
    """(table [positions][pairs][2] float32, pos [T][axes] int32, pairs of each axis)"""
    pairs = case["dim"] // 2
    if case["axes"] == 1:
        axis_pairs, pos = [pairs], pos0[:, None]
    else:
        h, w = case["height"], case["width"]
        a = pairs // 3
        axis_pairs = [pairs - 2 * a, a, a]
        pos = torch.stack([pos0 // (h * w), pos0 // w % h, pos0 % w], 1)
    freq = torch.cat([10000.0 ** (-torch.arange(n, device=DEV, dtype=torch.float64) / n) for n in axis_pairs])
    angle = torch.arange(int(pos.max()) + 1, device=DEV, dtype=torch.float64)[:, None] * freq
    table = torch.stack([angle.cos(), angle.sin()], -1).float()
    return table, pos.to(torch.int32).contiguous(), axis_pairs


def _gain(g, dim):
    return (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(torch.bfloat16)


def _lengths(case):
    """query and cache lengths of the sequences: spread evenly over their ranges, in a mixed order"""
    n = case["seqs"]
    i = np.arange(n) * 37 % n if n % 37 else np.arange(n)
    f = i / max(1, n - 1)
    q = np.round(case["q_min"] + (case["q_max"] - case["q_min"]) * (1 - f)).astype(np.int64)
    kv = np.round(case["kv_min"] + (case["kv_max"] - case["kv_min"]) * f).astype(np.int64)
    if n == 1:
        q[:], kv[:] = case["q_max"], case["kv_max"]
    return q, kv


def prepare(case, seed):
    def pool(g, n_pages, heads, page, dim):
        """a cache that holds keys and values: dict of codes uint8 [pages][heads][page][dim/2] and meta int16 [..][dim/32]"""
        out = {}
        for what in ("k", "v"):
            codes = torch.empty(n_pages, heads, page, dim // 2, dtype=torch.uint8, device=DEV)
            meta = torch.empty(n_pages, heads, page, dim // 32, dtype=torch.int16, device=DEV)
            step = max(1, (1 << 24) // (heads * page * dim))
            for p in range(0, n_pages, step):
                m = min(step, n_pages - p)
                x = torch.randn(m, heads, page, dim, generator=g, device=DEV)
                x *= torch.exp(0.3 * torch.randn(m, heads, page, 1, generator=g, device=DEV))
                x[..., 5::37] *= 4                                                       # channels that stand out
                codes[p:p + m], meta[p:p + m] = _pack(*_encode(x))
            out[what + "_codes"], out[what + "_meta"] = codes, meta
        return out

    g = _gen(seed)
    dim = case["dim"]
    if case["op"] in ("rotate", "append"):
        rotate = case["op"] == "rotate"
        hq, hk = case["q_heads"], case["k_heads" if rotate else "kv_heads"]
        seqs = 1 if rotate else case["seqs"]
        n = case["tokens"] * seqs
        x = _projection(g, n, (hq + 2 * hk) * dim).view(n, hq + 2 * hk, dim)      # the packed result of one projection
        start = 0 if case["axes"] == 3 else 1000
        table, pos, axis_pairs = _rope(case, start + torch.arange(n, device=DEV) % case["tokens"])
        s = dict(case=case, q=x[:, :hq], k=x[:, hq:hq + hk], v=x[:, hq + hk:], table=table, pos=pos, axis_pairs=axis_pairs,
                 interleaved=case["interleaved"], q_gain=_gain(g, dim), k_gain=_gain(g, dim))
        if rotate:
            return s
        page = case["page"]
        per = -(-(case["tokens"] + page) // page)
        pages = torch.randperm(per * seqs, generator=g, device=DEV).view(seqs, per)
        at = torch.arange(case["tokens"], device=DEV)[None, :] + (torch.arange(seqs, device=DEV) * 7 % page)[:, None]
        slot = torch.gather(pages, 1, at // page) * page + at % page
        slot = slot.view(-1).to(torch.int64)
        if seqs > 1:
            slot[n - n // 50:] = -1                                                  # rows that pad the batch
        s["slot"] = slot
        s["cache"] = pool(g, per * seqs, hk, page, dim)
        return s
    q_len, kv_len = _lengths(case)
    page = case["page"]
    need = -(-kv_len // page)
    n_pages = int(need.sum()) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(case["seqs"], max(1, int(need.max())), dtype=torch.int32, device=DEV)
    first = np.concatenate([[0], np.cumsum(need)])
    for i in range(case["seqs"]):
        table[i, :need[i]] = perm[first[i]:first[i + 1]]
    total = int(q_len.sum())
    q = torch.randn(total, case["q_heads"], dim, generator=g, device=DEV)
    q *= torch.exp(0.5 * torch.randn(total, case["q_heads"], 1, generator=g, device=DEV)) * 1.5    # from flat to peaked rows
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a.astype(np.int32))).to(DEV)  # noqa: E731
    return dict(case=case, q=q.to(torch.bfloat16), cache=pool(g, n_pages, case["kv_heads"], page, dim), page_table=table,
                kv_len=dev(kv_len), q_start=dev(np.concatenate([[0], np.cumsum(q_len)])), max_q=int(q_len.max()),
                max_kv=int(kv_len.max()), scale=dim ** -0.5, causal=case["causal"], window=case["window"])


# ---------------------------------------------------------------------------------------------------- plain forms

def _norm_rotate(x, gain, table, pos, axis_pairs, interleaved):
    """float32, every operation rounded once; the squares are added by folding every run of 8 channels in halves, then the runs
    of the row's two halves pairwise, then these sums (filled up with zeros to a power of two) in halves"""
    x = x.float()
    t, h, dim = x.shape
    s = (x * x).view(t, h, dim // 8, 8)
    s = s[..., :4] + s[..., 4:]
    s = s[..., :2] + s[..., 2:]
    s = s[..., 0] + s[..., 1]
    s = s[..., :dim // 16] + s[..., dim // 16:]
    s = torch.nn.functional.pad(s, (0, 16 - dim // 16))
    s = s[..., :8] + s[..., 8:]
    s = s[..., :4] + s[..., 4:]
    s = s[..., :2] + s[..., 2:]
    s = s[..., :1] + s[..., 1:]
    r = torch.reciprocal(torch.sqrt(s * float(np.float32(1.0 / dim)) + float(np.float32(EPS))))
    y = (x * r) * gain.float()
    axis = torch.repeat_interleave(torch.arange(len(axis_pairs), device=x.device), torch.tensor(axis_pairs, device=x.device))
    cs = table[pos.long()[:, axis], torch.arange(dim // 2, device=x.device)][:, None]
    c, sn = cs[..., 0], cs[..., 1]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :dim // 2], y[..., dim // 2:])
    u, w = a * c - b * sn, b * c + a * sn
    return torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)


def _run_rotate(s):
    if own:
        f = _fb4()
        rope = _module().Rope(s["table"], s["pos"], s["axis_pairs"], s["interleaved"])
        return f.qk_norm_rope(s["q"], s["k"], s["q_gain"], s["k_gain"], EPS, rope)
    a = (s["table"], s["pos"], s["axis_pairs"], s["interleaved"])
    return (_norm_rotate(s["q"], s["q_gain"], *a).to(torch.bfloat16), _norm_rotate(s["k"], s["k_gain"], *a).to(torch.bfloat16))


def _run_append(s):
    """q, and all that the cache holds afterwards, as the values its codes stand for (every FB4 value is a bfloat16 number)"""
    c = s["cache"]
    if own:
        f = _fb4()
        m = _module()
        cache = m.Cache(c["k_codes"], c["k_meta"], c["v_codes"], c["v_meta"])
        rope = m.Rope(s["table"], s["pos"], s["axis_pairs"], s["interleaved"])
        q = f.cache_append(cache, s["slot"], s["k"], s["v"], s["k_gain"], EPS, rope, q=s["q"], q_gain=s["q_gain"])
        return (q, *f.cache_values(cache, torch.bfloat16))
    a = (s["table"], s["pos"], s["axis_pairs"], s["interleaved"])
    q = _norm_rotate(s["q"], s["q_gain"], *a).to(torch.bfloat16)
    k = _values(*_encode(_norm_rotate(s["k"], s["k_gain"], *a)))
    v = _values(*_encode(s["v"].float()))
    page = c["k_codes"].shape[2]
    rows = s["slot"] >= 0
    at = s["slot"][rows]
    kc, vc = _unpack(c["k_codes"], c["k_meta"]), _unpack(c["v_codes"], c["v_meta"])
    kc[at // page, :, at % page] = k[rows]
    vc[at // page, :, at % page] = v[rows]
    return q, kc.to(torch.bfloat16), vc.to(torch.bfloat16)


def _run_attend(s):
    c = s["cache"]
    if own:
        m = _module()
        cache = m.Cache(c["k_codes"], c["k_meta"], c["v_codes"], c["v_meta"])
        return _fb4().cache_attention(s["q"], cache, s["page_table"], s["kv_len"], s["q_start"], s["max_q"], s["max_kv"],
                                      scale=s["scale"], causal=s["causal"], window=s["window"])
    q, page_table = s["q"], s["page_table"].long()
    total, hq, dim = q.shape
    b, hk = page_table.shape[0], c["k_codes"].shape[1]
    k = _unpack(c["k_codes"][page_table], c["k_meta"][page_table]).transpose(1, 2).reshape(b, hk, -1, dim)
    v = _unpack(c["v_codes"][page_table], c["v_meta"][page_table]).transpose(1, 2).reshape(b, hk, -1, dim)
    n, mq = k.shape[2], s["max_q"]
    q_len = (s["q_start"][1:] - s["q_start"][:-1]).long()
    kv_len = s["kv_len"].long()
    i = torch.arange(mq, device=q.device)
    rows = (s["q_start"][:-1].long()[:, None] + i).clamp(max=total - 1)
    qs = q[rows].float().view(b, mq, hk, hq // hk, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, dim)      # [b][hk][group * mq][dim]
    pos = (kv_len - q_len)[:, None] + i
    j = torch.arange(n, device=q.device)
    see = (j[None, None, :] < kv_len[:, None, None]).expand(b, mq, n)
    if s["causal"]:
        see = see & (j[None, None, :] <= pos[:, :, None])
    if s["window"]:
        see = see & (j[None, None, :] > pos[:, :, None] - s["window"])
    score = torch.matmul(qs, k.transpose(2, 3)).mul_(s["scale"]).view(b, hk, hq // hk, mq, n)
    score.masked_fill_(~see[:, None, None], float("-inf"))
    m = score.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = score.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, n), v).view(b, hk, hq // hk, mq, dim)
    o = torch.where(l > 0, o / l, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(b, mq, hq, dim)
    lse = (m + l.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(b, mq, hq)
    valid = i[None, :] < q_len[:, None]
    return o[valid].to(torch.bfloat16), lse[valid]


def run(state):
    return {"rotate": _run_rotate, "append": _run_append, "attend": _run_attend}[state["case"]["op"]](state)


def _module():
    from paper_2603_02883_b200 import fb4
    return fb4


def _fb4():
    """the context a program holds from its start"""
    if "ctx" not in _const:
        _const["ctx"] = _module().Fb4()
    return _const["ctx"]


# ---------------------------------------------------------------------------------------------------- work

def work(case):
    dim = case["dim"]
    if case["op"] != "attend":
        rotate = case["op"] == "rotate"
        hk = case["k_heads" if rotate else "kv_heads"]
        n = case["tokens"] * (1 if rotate else case["seqs"])
        if case["axes"] == 1:
            used = case["tokens"]
        else:
            used = max(case["width"], case["height"], -(-case["tokens"] // (case["height"] * case["width"])))
        side = n * case["axes"] * 4 + min(n * 3, used) * dim // 2 * 8
        if rotate:
            return {"bytes": n * (case["q_heads"] + hk) * dim * 4 + side, "flops": 9 * n * (case["q_heads"] + hk) * dim}
        page = case["page"]
        pool = case["seqs"] * -(-(case["tokens"] + page) // page) * page * hk * dim * 2
        # q through, k and v in, their blocks out; then the whole pool as values: its blocks in, two bytes a value out
        return {"bytes": n * case["q_heads"] * dim * 4 + n * hk * dim * 2 * (2 + 0.5625) + side + n * 8 + pool * 2.5625,
                "flops": 9 * n * (case["q_heads"] + hk) * dim + 12 * n * 2 * hk * dim}
    q_len, kv_len = _lengths(case)
    pairs = seen = 0
    for a, b in zip(q_len.tolist(), kv_len.tolist()):
        pos = b - a + np.arange(a)
        hi = np.minimum(pos + 1, b) if case["causal"] else np.full(a, b)
        lo = np.maximum(pos - case["window"] + 1, 0) if case["window"] else np.zeros(a, np.int64)
        n = np.maximum(hi - lo, 0)
        pairs += int(n.sum())
        seen += max(0, int(hi.max() - lo[n > 0].min())) if (n > 0).any() else 0
    total = int(q_len.sum())
    return {"bytes": total * case["q_heads"] * (dim * 4 + 4) + seen * case["kv_heads"] * dim * 2 * 0.5625 + 4 * len(q_len) * (2 + int(kv_len.max()) / case["page"]),
            "flops": 4 * pairs * case["q_heads"] * dim}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    def decode64(codes, meta):
        out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
        book = torch.tensor(BOOK, dtype=torch.float64, device=codes.device)
        for half in (0, 1):
            nib = (codes >> (4 * half)) & 15
            m = meta.to(torch.int64).repeat_interleave(16, dim=-1)
            mag = book[(m >> 8) & 31, (nib & 7).long()]
            out[..., half::2] = mag * torch.where(nib > 7, -1.0, 1.0) * torch.pow(2.0, ((m & 255) - 127).double())
        return out

    def quantized64(x):
        """x float64 [n][32] -> the values of its FB4 blocks"""
        book = torch.tensor(BOOK, dtype=torch.float64, device=x.device)
        top = x.abs().amax(1)
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -124)))
        e = torch.where(torch.pow(2.0, e) > top, e - 1, torch.where(torch.pow(2.0, e + 1) <= top, e + 1, e)).clamp(min=-124.0)
        unit = torch.pow(2.0, e - 3)[:, None]
        u = x.abs() / unit
        group = u.view(-1, 8, 4).amax(2)
        mid = torch.floor(group * 2) / 2 + 0.25
        best = torch.full_like(top, float("inf"))
        out = torch.zeros_like(x)
        for d in range(32):
            err = (mid[:, :, None] - book[d]).abs().amin(2).sum(1)
            allowed = torch.floor(u.amax(1)).clamp(min=8.0) == book[d, 7]
            better = allowed & (err < best)
            best = torch.where(better, err, best)
            edge = (book[d, 1:] + book[d, :-1]) / 2
            near = book[d][torch.bucketize(u, edge, right=True)]
            out = torch.where(better[:, None], near * unit * torch.where(torch.signbit(x), -1.0, 1.0).double(), out)
        return out

    def rotated64(x, gain, s):
        x = x.double()
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.double()
        out = torch.empty_like(y)
        at = 0
        dim = x.shape[-1]
        for axis, n in enumerate(s["axis_pairs"]):
            p = torch.arange(at, at + n, device=x.device)
            first, second = (2 * p, 2 * p + 1) if s["interleaved"] else (p, p + dim // 2)
            freq = 10000.0 ** (-torch.arange(n, device=x.device, dtype=torch.float64) / n)
            angle = (s["pos"][:, axis].double()[:, None] * freq)[:, None]
            out[..., first] = y[..., first] * torch.cos(angle) - y[..., second] * torch.sin(angle)
            out[..., second] = y[..., first] * torch.sin(angle) + y[..., second] * torch.cos(angle)
            at += n
        return out

    s = prepare(case, seed)
    if case["op"] == "rotate":
        return rotated64(s["q"], s["q_gain"], s), rotated64(s["k"], s["k_gain"], s)
    c = s["cache"]
    if case["op"] == "append":
        q = rotated64(s["q"], s["q_gain"], s)
        out = [q]
        for name, x in (("k", rotated64(s["k"], s["k_gain"], s)), ("v", s["v"].double())):
            held = decode64(c[name + "_codes"], c[name + "_meta"])
            new = torch.cat([quantized64(b) for b in x.reshape(-1, 32).split(1 << 20)]).view(x.shape)
            page = held.shape[2]
            rows = s["slot"] >= 0
            at = s["slot"][rows]
            held[torch.div(at, page, rounding_mode="floor"), :, at % page] = new[rows]
            out.append(held)
        return tuple(out)
    q_len, kv_len = _lengths(case)
    group = case["q_heads"] // case["kv_heads"]
    outs, lses, at = [], [], 0
    for i, (a, n) in enumerate(zip(q_len.tolist(), kv_len.tolist())):
        pages = s["page_table"][i, :-(-n // case["page"])].long()
        k = decode64(c["k_codes"][pages], c["k_meta"][pages]).transpose(0, 1).flatten(1, 2)[:, :n]
        v = decode64(c["v_codes"][pages], c["v_meta"][pages]).transpose(0, 1).flatten(1, 2)[:, :n]
        pos = n - a + torch.arange(a, device=DEV)
        j = torch.arange(n, device=DEV)
        hide = torch.zeros(a, n, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hide |= j > pos[:, None]
        if case["window"]:
            hide |= j <= pos[:, None] - case["window"]
        o = torch.zeros(a, case["q_heads"], case["dim"], dtype=torch.float64, device=DEV)
        lse = torch.zeros(a, case["q_heads"], dtype=torch.float64, device=DEV)
        for h in range(case["q_heads"]):
            z = (s["q"][at:at + a, h].double() @ k[h // group].T) * s["scale"]
            z = z.masked_fill(hide, float("-inf"))
            lse[:, h] = torch.logsumexp(z, 1)
            w = torch.exp(z - torch.where(torch.isinf(lse[:, h]), torch.zeros_like(lse[:, h]), lse[:, h])[:, None])
            o[:, h] = w @ v[h // group]
        outs.append(o)
        lses.append(lse)
        at += a
    return torch.cat(outs), torch.cat(lses)
