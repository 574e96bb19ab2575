"""Plain statements of the 8-bit cache, from include/fb4.h: its decode, the append (numpy), and attention over it in float64 (with the
error bounds of attend_ref, whose kernels' roundings are the same)."""
from types import SimpleNamespace

import numpy as np
import torch

import attend_ref
from paper_2603_02883_b200 import fb4


def decode64(codes, scale):
    """codes [..., tokens, D], scale [..., tokens / 16] -> float64"""
    e = scale.to(torch.int64).clamp(58, 185) - 127
    unit = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e.cpu()).to(codes.device)
    return (codes.double() - 128) * unit.repeat_interleave(16, -1)[..., None]


def attend64(q, cache, *args):
    """attend_ref.attend64 on an 8-bit cache"""
    view = SimpleNamespace(k_codes=cache.k, k_meta=cache.k_scale, v_codes=cache.v, v_meta=cache.v_scale)
    kept = attend_ref.decode64
    attend_ref.decode64 = decode64
    try:
        return attend_ref.attend64(q, view, *args)
    finally:
        attend_ref.decode64 = kept


def exponent(top):
    """the smallest e in [-69, 58] with top < 127.5 * 2^e"""
    e = -69
    while e < 58 and not top < 127.5 * 2.0 ** e:
        e += 1
    return e


def append(x, codes, scale, table, kv_len, q_start):
    """x float32 [T][H][D] after norm and rotation; codes [pages][H][page][D] and scale [pages][H][page / 16] are changed"""
    n_pages, H, page, D = codes.shape
    for b in range(len(kv_len)):
        n, kv, r0 = int(q_start[b + 1] - q_start[b]), int(kv_len[b]), int(q_start[b])
        first = max(kv - n, 0)
        for base in range(first // 16 * 16, kv if n else 0, 16):
            p = int(table[b, base // page])
            if p < 0 or p >= n_pages:
                continue
            lo, hi = max(first - base, 0), min(kv - base, 16)
            at, blk = base % page, base % page // 16
            rows = np.float64(x[r0 + base + lo - (kv - n): r0 + base + hi - (kv - n)])                 # [new][H][D]
            for h in range(H):
                e = exponent(np.abs(rows[:, h]).max())
                if lo:
                    held = min(max(int(scale[p, h, blk]), 58), 185) - 127
                    s = max(e, held)
                    c = codes[p, h, at:at + lo].astype(np.float64) - 128
                    codes[p, h, at:at + lo] = (np.rint(c * 2.0 ** (held - s)) + 128).astype(np.uint8)
                    e = s
                codes[p, h, at + lo:at + hi] = (np.clip(np.rint(rows[:, h] * 2.0 ** -e), -127, 127) + 128).astype(np.uint8)
                scale[p, h, blk] = e + 127


def random_cache(n_pages, heads, page, D, seed, lo=118, hi=124):
    """any codes, and scales between lo and hi"""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda a, b, *shape: torch.randint(a, b, shape, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    return fb4.Cache8(r(0, 256, n_pages, heads, page, D), r(lo, hi, n_pages, heads, page // 16), r(0, 256, n_pages, heads, page, D),
                      r(lo, hi, n_pages, heads, page // 16))


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def tables(q_len, kv_len, page, seed, spare=2):
    """(page_table with -7 behind the last page, number of pages, kv_len, q_start) on the device"""
    q_len, kv_len = np.asarray(q_len), np.asarray(kv_len)
    need = -(-kv_len // page)
    n_pages = int(need.sum()) + spare
    perm = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((len(kv_len), max(1, int(need.max()))), -7, np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    return i32(table), n_pages, i32(kv_len), i32(np.concatenate([[0], np.cumsum(q_len)]))


def setup(q_len, kv_len, Hq, Hk, D, page, seed=0, spread=1.5):
    table, n_pages, kv, qs = tables(q_len, kv_len, page, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = (torch.randn(int(sum(q_len)), Hq, D, generator=g, device="cuda") * spread).to(torch.bfloat16)
    return q, random_cache(n_pages, Hk, page, D, seed), table, kv, qs, max(q_len), max(kv_len)
