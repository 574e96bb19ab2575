"""Plain forms and measured cases of the operators of a decoding step: the step's plan, the append to an 8-bit cache, attention
over that cache, and products with FB4 weights.

Four operators, in the order a serving step uses them:
  plan     sequences keep their first keep[b] tokens and get new[b] more: pages go back to and come from a free list, and the rows
           of the step get their sequence, position and cache slot
  linear   y = x W^T + bias for a few rows x, W in FB4 blocks of 32 (the offline weight quantizer's output)
  append   q, k through RMS norm and rotation, then k and v to the pages of an 8-bit cache
  attend   softmax(scale * q k^T) v of the new tokens of several sequences over their pages of that cache

The 8-bit cache: the 16 tokens of a block share one power of two for each head, separately for k and v.  A value is
(code - 128) * 2^(scale - 127) with code in 1..255.  The exponent of new tokens is the smallest e in [-69, 58] with
max |x| < 127.5 * 2^e; tokens that a block holds already keep the larger of both exponents and are rounded to it if it is the new one.

FB4 (weights; block of 32 channels): e = floor(log2(max |x|)), element scale 2^(e-3); codes uint8 [..][K/2], low nibble first,
nibble = sign << 3 | index into the dialect's 8 magnitudes; meta int16 [..][K/32], bits 0-7 = e + 124, bits 8-12 = dialect.
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
        # a decoding step: every sequence one more token, nothing dropped: all latency
        dict(name="plan 64 x 1", op="plan", seqs=64, page=16, held=4000, drop=0, new_min=1, new_max=1, fresh=0, prompt=0, short=False, tight=False),
        # a large server: drafted tokens dropped and added, every 16th sequence has ended and a prompt takes its place
        dict(name="plan 2048, prompts", op="plan", seqs=2048, page=16, held=8191, drop=7, new_min=1, new_max=8, fresh=16, prompt=4097, short=False, tight=False),
        # one token through a square projection of the largest layer in the benchmark: a matrix-vector product
        dict(name="linear 1 x 12288 x 12288", op="linear", tokens=1, n=12288, k=12288, pad=0, bias=False),
        # a decoding batch through the first half of a feed-forward block: the largest
        dict(name="linear 16 x 24576 x 12288", op="linear", tokens=16, n=24576, k=12288, pad=0, bias=False),
        # drafted tokens of several sequences, sizes that no tile divides, a bias, rows with a stride
        dict(name="linear 61 x 6152 x 1568", op="linear", tokens=61, n=6152, k=1568, pad=40, bias=True),
        # one new token for each of 64 sequences, most of them into blocks that hold tokens
        dict(name="append 64 x 1", op="append", seqs=64, q_min=1, q_max=1, held=100, q_heads=32, kv_heads=8, dim=128, axes=1, interleaved=False, height=0, width=0, page=16),
        # ragged prompts behind a cached part, narrow heads, padded rows at the end of the batch
        dict(name="append 3 x 1365", op="append", seqs=3, q_min=700, q_max=1365, held=333, q_heads=16, kv_heads=4, dim=64, axes=1, interleaved=False, height=0, width=0, page=32),
        # a clip's keys and values at once: the largest
        dict(name="append a clip", op="append", seqs=1, q_min=32760, q_max=32760, held=0, q_heads=12, kv_heads=12, dim=128, axes=3, interleaved=True, height=30, width=52, page=64),
        # one token of one sequence over the longest cache
        dict(name="attend 1 over 75600", op="attend", seqs=1, q_min=1, q_max=1, kv_min=75600, kv_max=75600, q_heads=12, kv_heads=12, dim=128, page=64, causal=True, window=0),
        # a serving batch: 64 sequences of very different lengths, four query heads to a cache head
        dict(name="attend 64 x 1, ragged", op="attend", seqs=64, q_min=1, q_max=1, kv_min=131, kv_max=8191, q_heads=32, kv_heads=8, dim=128, page=16, causal=True, window=0),
        # prompts in chunks, causal against all that is cached; narrow heads
        dict(name="attend 4 x 1024, causal", op="attend", seqs=4, q_min=515, q_max=1024, kv_min=1024, kv_max=4096, q_heads=16, kv_heads=4, dim=64, page=32, causal=True, window=0),
        # a new frame over a cached clip, every token seeing all of it
        dict(name="attend a frame", op="attend", seqs=1, q_min=1560, q_max=1560, kv_min=32760, kv_max=32760, q_heads=12, kv_heads=12, dim=128, page=64, causal=False, window=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["plan", "linear", "linear", "append", "attend", "attend"])
    if op == "plan":
        seqs = _log(rng, 1, 2048)
        fresh = rng.choice([0, 0, 3, 16, 50])
        prompt = _log(rng, 1, max(1, min(32760, 500_000 * max(1, fresh) // seqs))) if fresh else 0
        new_max = _log(rng, 1, max(1, min(4096, 250_000 // seqs)))
        return dict(op=op, seqs=seqs, page=rng.choice([16, 32, 64, 128]), held=_log(rng, 1, 8191), drop=rng.choice([0, 0, 7, 300]),
                    new_min=rng.randint(0, new_max), new_max=new_max, fresh=fresh, prompt=prompt, short=rng.random() < 0.25, tight=rng.random() < 0.25)
    if op == "linear":
        k = 32 * _log(rng, 1, 512)
        return dict(op=op, tokens=_log(rng, 1, 64), n=_log(rng, 1, min(49152, 24576 * 12288 // k)), k=k, pad=8 * rng.choice([0, 0, 1, 5]), bias=rng.random() < 0.5)
    kv = rng.choice([1, 2, 4, 5, 8, 12, 16])
    group = rng.choice([1, 1, 2, 4, 7, 8])
    if kv * group > 40:
        group = 1
    if op == "append":
        dim = rng.choice([64, 96, 128, 128])
        axes = rng.choice([1, 3])
        most = max(64, 32760 * 27 * 128 // ((kv * group + kv * 2) * dim))
        seqs = _log(rng, 1, 64)
        q_max = _log(rng, 1, max(1, min(32760, most // seqs)))
        held = rng.choice([0, _log(rng, 1, max(1, min(2000, 32760 * 3 * 128 // (seqs * kv * dim))))])
        return dict(op=op, seqs=seqs, q_min=rng.randint(1, q_max), q_max=q_max, held=held, q_heads=kv * group, kv_heads=kv, dim=dim, axes=axes,
                    interleaved=rng.random() < 0.5, height=rng.randint(3, 48) if axes == 3 else 0, width=rng.randint(3, 80) if axes == 3 else 0,
                    page=rng.choice([16, 32, 64, 128]))
    dim = rng.choice([64, 128, 128])
    kind = rng.choice(["one", "few", "many"])
    seqs = _log(rng, 1, 96 if kind != "many" else 8)
    q_max = 1 if kind == "one" else _log(rng, 2, 24) if kind == "few" else _log(rng, 25, 2048)
    kv_max = min(75600, 75600 * 12 * 128 // (seqs * kv * dim), 500_000_000 // (seqs * q_max * kv * group))
    kv_max = _log(rng, 1, max(1, kv_max))
    kv_min = _log(rng, 1, kv_max)
    return dict(op=op, q_heads=kv * group, kv_heads=kv, dim=dim, seqs=seqs, q_min=rng.randint(1, q_max), q_max=q_max, kv_min=kv_min, kv_max=kv_max,
                page=rng.choice([16, 32, 64, 128]), causal=rng.random() < 0.7, window=rng.choice([0, 0, 0, _log(rng, 1, 5000)]))


# ---------------------------------------------------------------------------------------------------- the formats, plainly

_const = {}


def _tables():
    """qerr[bin][dialect] in quarter units, qvalue[dialect][bin], stage1[bin][dialect], book[dialect][index]"""
    if "t" not in _const:
        book = np.array(BOOK, np.int64)
        k = np.arange(32)
        index = ((book[:, None, 1:] + book[:, None, :-1]) <= k[None, :, None]).sum(2)             # [dialect][bin]
        err = np.abs(2 * k[None, :] + 1 - 4 * np.take_along_axis(book, index, 1))
        first = book[None, :, 7] == np.maximum(8, k[:, None] // 2)
        _const["t"] = tuple(map(lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV),
                                (err.T.astype(np.float32), index, first, book.astype(np.float32))))
    return _const["t"]


def _fb4_encode(x):
    """x float32 [..., 32 n] -> codes uint8 [..., 16 n], meta int16 [..., n]"""
    qerr, qvalue, stage1, _ = _tables()
    b = x.reshape(-1, 32)
    top = b.abs().amax(1)
    e = torch.where(top == 0, torch.full_like(top, -124).int(), (torch.frexp(top).exponent - 1).clamp(-124, 127))
    bins = torch.floor(torch.ldexp(b.abs(), (4 - e)[:, None])).to(torch.int64).clamp_(max=31)
    err = qerr[bins.view(-1, 8, 4).amax(2)].sum(1)
    key = torch.where(stage1[bins.amax(1)], err * 32 + torch.arange(32, device=x.device), float("inf"))
    did = key.amin(1).to(torch.int64) % 32
    code = qvalue.view(-1)[did[:, None] * 32 + bins] + 8 * torch.signbit(b).to(torch.int64)
    code = code.to(torch.uint8).view(*x.shape[:-1], -1, 2)
    meta = ((e + 124) | (did << 8)).to(torch.int16)
    return (code[..., 0] | (code[..., 1] << 4)).contiguous(), meta.view(*x.shape[:-1], -1)


def _fb4_values(codes, meta):
    """what codes stand for, float32 (exact)"""
    book = _tables()[3]
    c = torch.stack([codes & 15, codes >> 4], -1).view(*meta.shape, 32).to(torch.int32)
    m = meta.to(torch.int32)
    mag = book.view(-1)[((m >> 8) & 31)[..., None] * 8 + (c & 7)]
    v = torch.ldexp(torch.where(c >= 8, -mag, mag), ((m & 255) - 127)[..., None])
    return v.flatten(-2)


def _exponent(top):
    """the smallest e in [-69, 58] with top < 127.5 * 2^e"""
    m, x = torch.frexp(top)                                               # top = m * 2^x, m in [0.5, 1)
    e = x - 7 + (m >= 255.0 / 256.0).to(x.dtype)
    return torch.where(top == 0, torch.full_like(e, -69), e).clamp(-69, 58)


def _int8_values(codes, scale):
    """codes uint8 [pages][heads][tokens][D], scale uint8 [pages][heads][tokens / 16] -> float32 (exact)"""
    e = (scale.to(torch.int32) - 127)[..., None, None]
    c = (codes.to(torch.float32) - 128).unflatten(2, (-1, 16))
    return torch.ldexp(c, e).flatten(2, 3)


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
    a = pairs // 3
    axis_pairs = [pairs] if case["axes"] == 1 else [pairs - 2 * a, a, a]
    h, w = max(1, case["height"]), max(1, case["width"])
    pos = pos0[:, None] if case["axes"] == 1 else torch.stack([pos0 // (h * w), pos0 // w % h, pos0 % w], 1)
    freq = torch.cat(list(map(lambda n: 10000.0 ** (-torch.arange(n, device=DEV, dtype=torch.float64) / n), axis_pairs)))
    angle = torch.arange(int(pos.max()) + 1, device=DEV, dtype=torch.float64)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float(), pos.to(torch.int32).contiguous(), axis_pairs


def _gain(g, dim):
    return (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(torch.bfloat16)


def _lengths(case):
    """query and cache lengths of the sequences: spread evenly over their ranges, in a mixed order"""
    n = case["seqs"]
    i = np.arange(n) * 37 % n if n % 37 else np.arange(n)
    f = i / max(1, n - 1)
    q = np.round(case["q_min"] + (case["q_max"] - case["q_min"]) * (1 - f)).astype(np.int64)
    if case["op"] == "append":
        kv = q + (np.arange(n) * 7919 + 5) % (case["held"] + 1)
    else:
        kv = np.round(case["kv_min"] + (case["kv_max"] - case["kv_min"]) * f).astype(np.int64)
    if n == 1 and case["op"] == "attend":
        q[:], kv[:] = case["q_max"], case["kv_max"]
    return q, kv


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(np.int32))).to(DEV)


def _plan_lengths(case, seed):
    """what the sequences hold, keep and get; another seed deals the same lengths out to other sequences"""
    r = np.random.RandomState(1)
    n = case["seqs"]
    held = r.randint(0, case["held"] + 1, n)
    keep = np.maximum(held - r.randint(0, case["drop"] + 1, n), 0)
    new = r.randint(case["new_min"], case["new_max"] + 1, n)
    if case["fresh"]:
        at = np.arange(n) % case["fresh"] == case["fresh"] - 1
        keep = np.where(at, 0, keep)
        new = np.where(at, r.randint(1, case["prompt"] + 1, n), new)
    order = np.random.RandomState(seed % (1 << 31)).permutation(n)
    return held[order], keep[order], new[order]


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "plan":
        page = case["page"]
        held, keep, new = _plan_lengths(case, seed)
        pages, kept, want = -(-held // page), -(-keep // page), -(-(keep + new) // page)
        need, back = int((want - kept).sum()), int((pages - kept).sum())
        n_free = max(0, need // 2 - back) if case["short"] else max(0, need - back) + 7
        n_pages = int(pages.sum()) + n_free
        perm = torch.randperm(max(1, n_pages), generator=g, device=DEV).to(torch.int32)
        table = torch.full((case["seqs"], max(1, int(max(pages.max(), want.max())))), -1, dtype=torch.int32, device=DEV)
        filled = torch.arange(table.shape[1], device=DEV)[None] < _dev(pages)[:, None]
        table[filled] = perm[:int(pages.sum())]
        free = torch.full((max(1, n_pages),), -1, dtype=torch.int32, device=DEV)
        free[:n_free] = perm[int(pages.sum()):int(pages.sum()) + n_free]
        total = int(new.sum())
        return dict(case=case, page_table=table, kv_len=_dev(held), free_pages=free, n_free=_dev([n_free]), keep=_dev(keep), new=_dev(new),
                    rows=max(1, total * 9 // 10) if case["tight"] else total + total // 50)
    if case["op"] == "linear":
        n, k, t = case["n"], case["k"], case["tokens"]
        codes = torch.empty(n, k // 2, dtype=torch.uint8, device=DEV)
        meta = torch.empty(n, k // 32, dtype=torch.int16, device=DEV)
        step = max(1, (1 << 24) // k)
        for r in range(0, n, step):
            w = torch.randn(min(step, n - r), k, generator=g, device=DEV)
            w *= k ** -0.5 * torch.exp(0.2 * torch.randn(w.shape[0], 1, generator=g, device=DEV))
            codes[r:r + step], meta[r:r + step] = _fb4_encode(w)
        x = _projection(g, t, k + case["pad"])[:, :k]
        bias = (0.1 * torch.randn(n, generator=g, device=DEV)).to(torch.bfloat16) if case["bias"] else None
        return dict(case=case, x=x, codes=codes, meta=meta, bias=bias)

    def pool(n_pages, heads, page, dim):
        """a cache that holds keys and values: codes uint8 [pages][heads][page][dim], scales uint8 [pages][heads][page / 16]"""
        out = {}
        for what in ("k", "v"):
            codes = torch.empty(n_pages, heads, page, dim, dtype=torch.uint8, device=DEV)
            scale = torch.empty(n_pages, heads, page // 16, dtype=torch.uint8, device=DEV)
            step = max(1, (1 << 24) // (heads * page * dim))
            for p in range(0, n_pages, step):
                m = min(step, n_pages - p)
                x = torch.randn(m, heads, page, dim, generator=g, device=DEV)
                x *= torch.exp(0.3 * torch.randn(m, heads, page, 1, generator=g, device=DEV))
                x[..., 5::37] *= 4                                                       # channels that stand out
                b = x.unflatten(2, (-1, 16))
                e = _exponent(b.abs().amax((3, 4)))
                codes[p:p + m] = (torch.round(torch.ldexp(b, -e[..., None, None])).clamp(-127, 127) + 128).to(torch.uint8).flatten(2, 3)
                scale[p:p + m] = (e + 127).to(torch.uint8)
            out[what], out[what + "_scale"] = codes, scale
        return out

    dim, page = case["dim"], case["page"]
    q_len, kv_len = _lengths(case)
    need = -(-kv_len // page)
    n_pages = int(need.sum()) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(case["seqs"], max(1, int(need.max())), dtype=torch.int32, device=DEV)
    first = np.concatenate([[0], np.cumsum(need)])
    for i in range(case["seqs"]):
        table[i, :need[i]] = perm[first[i]:first[i + 1]]
    total = int(q_len.sum())
    s = dict(case=case, cache=pool(n_pages, case["kv_heads"], page, dim), page_table=table, kv_len=_dev(kv_len),
             q_start=_dev(np.concatenate([[0], np.cumsum(q_len)])), max_q=int(q_len.max()), total=total)
    if case["op"] == "append":
        n = total + (total // 50 if case["seqs"] > 1 else 0)                                # rows that pad the batch
        hq, hk = case["q_heads"], case["kv_heads"]
        x = _projection(g, n, (hq + 2 * hk) * dim).view(n, hq + 2 * hk, dim)              # the packed result of one projection
        at = np.concatenate([np.arange(b - a, b) for a, b in zip(q_len.tolist(), kv_len.tolist())] + [np.zeros(n - total, np.int64)])
        rope, pos, axis_pairs = _rope(case, _dev(at).long())
        return s | dict(q=x[:, :hq], k=x[:, hq:hq + hk], v=x[:, hq + hk:], table=rope, pos=pos, axis_pairs=axis_pairs,
                        interleaved=case["interleaved"], q_gain=_gain(g, dim), k_gain=_gain(g, dim))
    q = torch.randn(total, case["q_heads"], dim, generator=g, device=DEV)
    q *= torch.exp(0.5 * torch.randn(total, case["q_heads"], 1, generator=g, device=DEV)) * 1.5    # from flat to peaked rows
    return s | dict(q=q.to(torch.bfloat16), max_kv=int(kv_len.max()), scale=dim ** -0.5, causal=case["causal"], window=case["window"])


# ---------------------------------------------------------------------------------------------------- plain forms

def _run_plan(s):
    """the tables, lengths and free list after the step (all of them the state's own: planning the same step again gives the same),
    and the step's rows"""
    page = s["case"]["page"]
    table, kv_len, free, n_free = s["page_table"], s["kv_len"], s["free_pages"], s["n_free"]
    if own:
        pages = _module().PageTables(table, kv_len, free, n_free, page)
        plan = _fb4().cache_plan(pages, s["new"], s["rows"], keep=s["keep"])
        return table, kv_len, free, n_free, plan.q_start, plan.slot, plan.pos
    n, most = table.shape
    seq = torch.arange(n, device=DEV)
    held = kv_len.long().clamp(0, most * page)
    keep = torch.minimum(s["keep"].long().clamp(min=0), held)
    new = s["new"].long().clamp(min=0)
    up = lambda x: torch.div(x + page - 1, page, rounding_mode="floor")  # noqa: E731
    kept = up(keep)

    def flat(count):
        """(sequence, place among its own) of every one of `count` things of the sequences in order"""
        b = torch.repeat_interleave(seq, count)
        return b, torch.arange(b.numel(), device=DEV) - (count.cumsum(0) - count)[b]

    # pages given back, the first on top
    back = up(held) - kept
    top = n_free.long() + back.sum()
    b, i = flat(back)
    free[top - 1 - torch.arange(b.numel(), device=DEV)] = table[b, kept[b] + i]
    # who is served: what its table has room for, as long as pages and rows last
    new = torch.where(keep + new <= most * page, new, torch.zeros_like(new))
    need = up(keep + new) - kept
    served = (need.cumsum(0) <= top) & (new.cumsum(0) <= s["rows"])
    new = torch.where(served, new, torch.zeros_like(new))
    need = torch.where(served, need, torch.zeros_like(need))
    b, i = flat(need)
    table[b, kept[b] + i] = free[top - 1 - torch.arange(b.numel(), device=DEV)]
    kv_len.copy_(keep + new)
    n_free.copy_(top - need.sum())
    # the rows
    q_start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), new.cumsum(0)])
    b, i = flat(new)
    pos = torch.zeros(s["rows"], dtype=torch.int64, device=DEV)
    slot = torch.full((s["rows"],), -1, dtype=torch.int64, device=DEV)
    p = keep[b] + i
    pos[:b.numel()] = p
    slot[:b.numel()] = table[b, torch.div(p, page, rounding_mode="floor")].long() * page + p % page
    return table, kv_len, free, n_free, q_start.to(torch.int32), slot, pos.to(torch.int32)


def _run_linear(s):
    if own:
        w = _module().Quantized(s["codes"], s["meta"])
        return _fb4().linear(s["x"], w, bias=s["bias"])
    y = torch.matmul(s["x"].float(), _fb4_values(s["codes"], s["meta"]).t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(torch.bfloat16)


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


def _run_append(s):
    """q, and all that the cache holds afterwards, as the values its codes stand for (each of them a bfloat16 number)"""
    c, total = s["cache"], s["total"]
    if own:
        f, m = _fb4(), _module()
        cache = m.Cache8(c["k"], c["k_scale"], c["v"], c["v_scale"])
        rope = m.Rope(s["table"], s["pos"], s["axis_pairs"], s["interleaved"])
        q = f.cache8_append(cache, s["k"], s["v"], s["page_table"], s["kv_len"], s["q_start"], s["max_q"], s["k_gain"], EPS, rope, q=s["q"],
                            q_gain=s["q_gain"])
        return (q[:total], *f.cache8_values(cache, torch.bfloat16))
    a = (s["table"], s["pos"][:total], s["axis_pairs"], s["interleaved"])
    page = s["case"]["page"]
    q_len = (s["q_start"][1:] - s["q_start"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(q_len.numel(), device=DEV), q_len)
    place = s["kv_len"].long()[b] - q_len[b] + torch.arange(total, device=DEV) - s["q_start"].long()[b]
    block = s["page_table"].long()[b, place // page] * (page // 16) + place % page // 16             # of 16 tokens

    def write(x, codes, scale):
        """x float32 [total][heads][dim]"""
        n_pages, heads, _, dim = codes.shape
        held = codes.view(n_pages, heads, -1, 16, dim).transpose(1, 2).reshape(-1, heads, 16, dim)   # [block][head][token][dim]
        old = scale.transpose(1, 2).reshape(-1, heads).to(torch.int32) - 127
        top = torch.zeros(old.shape, device=DEV).index_reduce_(0, block, x.abs().amax(2), "amax")
        first = torch.full((old.shape[0],), 16, device=DEV).index_reduce_(0, block, place % 16, "amin")
        e = torch.where((first > 0)[:, None], torch.maximum(_exponent(top), old), _exponent(top))
        e = torch.where((first < 16)[:, None], e, old)
        fewer = torch.round(torch.ldexp(held.float() - 128, (old - e)[..., None, None]))
        before = torch.arange(16, device=DEV)[None] < first[:, None]                                 # tokens that stay
        out = torch.where(before[:, None, :, None], fewer, held.float() - 128)
        out[block, :, place % 16] = torch.round(torch.ldexp(x, -e[block][..., None])).clamp(-127, 127)
        back = lambda t: t.unflatten(0, (n_pages, -1)).transpose(1, 2)  # noqa: E731
        codes.copy_((back(out) + 128).to(torch.uint8).flatten(2, 3))
        scale.copy_((back(e) + 127).to(torch.uint8))
        return _int8_values(codes, scale).to(torch.bfloat16)

    q = _norm_rotate(s["q"][:total], s["q_gain"], *a).to(torch.bfloat16)
    k = write(_norm_rotate(s["k"][:total], s["k_gain"], *a), c["k"], c["k_scale"])
    return q, k, write(s["v"][:total].float(), c["v"], c["v_scale"])


def _run_attend(s):
    c = s["cache"]
    if own:
        cache = _module().Cache8(c["k"], c["k_scale"], c["v"], c["v_scale"])
        return _fb4().cache8_attention(s["q"], cache, s["page_table"], s["kv_len"], s["q_start"], s["max_q"], s["max_kv"],
                                       scale=s["scale"], causal=s["causal"], window=s["window"])
    q, page_table = s["q"], s["page_table"].long()
    total, hq, dim = q.shape
    b, hk = page_table.shape[0], c["k"].shape[1]
    spread = lambda name: _int8_values(c[name][page_table].flatten(0, 1), c[name + "_scale"][page_table].flatten(0, 1)).unflatten(0, (b, -1)).transpose(1, 2).reshape(b, hk, -1, dim)  # noqa: E731
    k, v = spread("k"), spread("v")
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
    return {"plan": _run_plan, "linear": _run_linear, "append": _run_append, "attend": _run_attend}[state["case"]["op"]](state)


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
    if case["op"] == "plan":
        n, page = case["seqs"], case["page"]
        held, keep, new = _plan_lengths(case, 1)
        rows = int(new.sum())
        moved = int((-(-held // page) + -(-(keep + new) // page) - 2 * -(-keep // page)).sum())
        # lengths in and out, pages moved from one list to the other, a slot and a position a row, the pages of the new tokens
        return {"bytes": n * 20 + moved * 8 + rows * (12 + 4 / page), "flops": rows * 4 + n * 8}
    if case["op"] == "linear":
        t, n, k = case["tokens"], case["n"], case["k"]
        return {"bytes": n * k * 0.5625 + t * k * 2 + t * n * 2 + (n * 2 if case["bias"] else 0), "flops": 2 * t * n * k}
    dim = case["dim"]
    q_len, kv_len = _lengths(case)
    total = int(q_len.sum())
    if case["op"] == "append":
        hq, hk, page = case["q_heads"], case["kv_heads"], case["page"]
        used = int(kv_len.max()) if case["axes"] == 1 else max(case["width"], case["height"], -(-int(kv_len.max()) // (case["height"] * case["width"])))
        side = total * case["axes"] * 4 + min(total * 3, used) * dim // 2 * 8
        pool = (int((-(-kv_len // page)).sum()) + 3) * page * hk * dim * 2
        # q through, k and v in, their codes out; then the whole pool as values: its codes in, two bytes a value out
        return {"bytes": total * hq * dim * 4 + total * hk * dim * 2 * 3 + side + pool * (3 + 1 / (16 * dim)),
                "flops": 9 * total * (hq + hk) * dim + 3 * total * 2 * hk * dim}
    pairs = seen = 0
    for a, b in zip(q_len.tolist(), kv_len.tolist()):
        pos = b - a + np.arange(a)
        hi = np.minimum(pos + 1, b) if case["causal"] else np.full(a, b)
        lo = np.maximum(pos - case["window"] + 1, 0) if case["window"] else np.zeros(a, np.int64)
        n = np.maximum(hi - lo, 0)
        pairs += int(n.sum())
        seen += max(0, int(hi.max() - lo[n > 0].min())) if (n > 0).any() else 0
    return {"bytes": total * case["q_heads"] * (dim * 4 + 4) + seen * case["kv_heads"] * 2 * (dim + 1 / 16) + 4 * len(q_len) * (2 + int(kv_len.max()) / case["page"]),
            "flops": 4 * pairs * case["q_heads"] * dim}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    powers = torch.tensor([2.0 ** e for e in range(-300, 301)], dtype=torch.float64, device=DEV)
    two_to = lambda e: powers[e.long() + 300]  # noqa: E731  (torch.pow is not exact here)
    if case["op"] == "plan":                            # sequence by sequence, as one would by hand
        page, rows = case["page"], s["rows"]
        table, free = s["page_table"].cpu().numpy().copy(), s["free_pages"].cpu().numpy().copy()
        held, keep, new = (s[x].cpu().numpy().astype(np.int64) for x in ("kv_len", "keep", "new"))
        stack = free[:int(s["n_free"])].tolist()
        back = np.concatenate([table[b, -(-keep[b] // page):-(-held[b] // page)] for b in range(len(held))])
        stack += back[::-1].tolist()
        free[:len(stack)] = stack
        kv, start, slot, pos, asked_pages, asked_rows = [], [0], [], [], 0, 0
        avail = len(stack)
        for b in range(len(held)):
            n, have = int(new[b]), -(-int(keep[b]) // page)
            n = n if keep[b] + n <= table.shape[1] * page else 0
            asked_pages += -(-(int(keep[b]) + n) // page) - have
            asked_rows += n
            if asked_pages > avail or asked_rows > rows:
                n = 0
            for at in range(have, -(-(int(keep[b]) + n) // page)):
                table[b, at] = stack.pop()
            p = keep[b] + np.arange(n)
            slot.append(table[b, p // page].astype(np.int64) * page + p % page)
            pos.append(p)
            kv.append(int(keep[b]) + n)
            start.append(start[-1] + n)
        rest = rows - start[-1]
        out = (table, np.array(kv, np.int32), free, np.array([len(stack)], np.int32), np.array(start, np.int32),
               np.concatenate(slot + [np.full(rest, -1, np.int64)]), np.concatenate(pos + [np.zeros(rest, np.int64)]).astype(np.int32))
        return tuple(torch.from_numpy(a) for a in out)
    if case["op"] == "linear":
        book = torch.tensor(BOOK, dtype=torch.float64, device=DEV)
        x = s["x"].double()
        parts = []
        step = max(1, (1 << 25) // case["k"])
        for r in range(0, case["n"], step):
            codes, meta = s["codes"][r:r + step], s["meta"][r:r + step].to(torch.int64).repeat_interleave(16, dim=-1)
            w = torch.empty(codes.shape[0], case["k"], dtype=torch.float64, device=DEV)
            for half in (0, 1):
                nib = (codes >> (4 * half)) & 15
                w[:, half::2] = book[(meta >> 8) & 31, (nib & 7).long()] * torch.where(nib > 7, -1.0, 1.0) * two_to((meta & 255) - 127)
            parts.append(x @ w.T)
        y = torch.cat(parts, 1)
        return y if s["bias"] is None else y + s["bias"].double()

    def decode64(codes, scale):
        return (codes.double() - 128) * two_to(scale.long() - 127).repeat_interleave(16, dim=2)[..., None]

    def rotated64(x, gain):
        x = x.double()
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.double()
        out = torch.empty_like(y)
        at = 0
        dim = x.shape[-1]
        for axis, n in enumerate(s["axis_pairs"]):
            p = torch.arange(at, at + n, device=x.device)
            first, second = (2 * p, 2 * p + 1) if s["interleaved"] else (p, p + dim // 2)
            freq = 10000.0 ** (-torch.arange(n, device=x.device, dtype=torch.float64) / n)
            angle = (s["pos"][:x.shape[0], axis].double()[:, None] * freq)[:, None]
            out[..., first] = y[..., first] * torch.cos(angle) - y[..., second] * torch.sin(angle)
            out[..., second] = y[..., first] * torch.sin(angle) + y[..., second] * torch.cos(angle)
            at += n
        return out

    c, page = s["cache"], case["page"]
    q_len, kv_len = _lengths(case)
    if case["op"] == "append":
        out = [rotated64(s["q"][:s["total"]], s["q_gain"])]
        for name, x in (("k", rotated64(s["k"][:s["total"]], s["k_gain"])), ("v", s["v"][:s["total"]].double())):
            held = decode64(c[name], c[name + "_scale"])
            unit = two_to(c[name + "_scale"].long() - 127)
            at = 0
            for i, (a, n) in enumerate(zip(q_len.tolist(), kv_len.tolist())):
                lo = (n - a) // 16 * 16                                                    # the first block that changes
                hi = -(-n // 16) * 16
                pages = s["page_table"][i].long()
                where = torch.arange(lo, hi, device=DEV)
                pg, in_page = pages[where // page], where % page
                vals = held[pg, :, in_page].clone()                                         # [tokens][heads][dim]
                stays = where < n - a
                fresh = (where >= n - a) & (where < n)
                vals[fresh] = x[at:at + a]
                top = torch.where(fresh[:, None], vals.abs().amax(2), torch.zeros_like(vals[..., 0])).unflatten(0, (-1, 16)).amax(1)
                e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -75) / 127.5))
                e = torch.where(top >= 127.5 * two_to(e), e + 1, torch.where(top < 127.5 * two_to(e - 1), e - 1, e))
                step = two_to(e.clamp(-69, 58))
                if stays.any():
                    step[0] = torch.maximum(step[0], unit[pg[0], :, in_page[0] // 16])
                step = step.repeat_interleave(16, dim=0)[..., None]
                new = torch.round(vals / step).clamp(-127, 127) * step
                keep = stays | fresh
                behind = (vals / unit[pg, :, in_page // 16][..., None]) * step              # what lies behind the new tokens keeps its codes
                held[pg, :, in_page] = torch.where(keep[:, None, None], new, behind)
                at += a
            out.append(held)
        return tuple(out)
    group = case["q_heads"] // case["kv_heads"]
    outs, lses, at = [], [], 0
    for i, (a, n) in enumerate(zip(q_len.tolist(), kv_len.tolist())):
        pages = s["page_table"][i, :-(-n // page)].long()
        k = decode64(c["k"][pages], c["k_scale"][pages]).transpose(0, 1).flatten(1, 2)[:, :n]
        v = decode64(c["v"][pages], c["v_scale"][pages]).transpose(0, 1).flatten(1, 2)[:, :n]
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
