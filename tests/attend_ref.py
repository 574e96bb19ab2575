"""Plain references of the attention-side operators: the stated float32 order of the norm and the rotation (numpy), and
masked attention over decoded cache pages in float64 (torch), with the error that the kernels' roundings allow."""
from __future__ import annotations

import numpy as np
import torch

from paper_2603_02883_b200 import synth

BOOK = synth.STANDIN_FORMATBOOK


def bf16_to_f32(bits):
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32)


def norm_rotate_f32(x, gain, eps, rope):
    """x float32 [T][H][D] -> float32, in the order include/fb4.h states at fb4_qk_norm_rope.  rope: None or (table, pos,
    axis_pairs, interleaved)"""
    x = np.asarray(x, np.float32)
    T, H, D = x.shape
    y = x
    if gain is not None:
        s = (x * x).reshape(T, H, D // 8, 8)
        s = s[..., :4] + s[..., 4:]
        s = s[..., :2] + s[..., 2:]
        s = s[..., 0] + s[..., 1]
        s = s[..., :D // 16] + s[..., D // 16:]
        n = 1
        while n < D // 16:
            n *= 2
        s = np.concatenate([s, np.zeros((T, H, n - D // 16), np.float32)], -1)
        while n > 1:
            n //= 2
            s = s[..., :n] + s[..., n:]
        t = s * np.float32(1.0 / D) + np.float32(eps)
        r = (np.float32(1.0) / np.sqrt(t)).astype(np.float32)
        y = (x * r) * np.asarray(gain, np.float32)
    if rope is None:
        return y
    table, pos, axis_pairs, interleaved = rope
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    p = pos.reshape(T, len(axis_pairs))[:, axis]
    p = np.where((p < 0) | (p >= table.shape[0]), 0, p)
    cs = table[p, np.arange(D // 2)][:, None]
    c, sn = cs[..., 0], cs[..., 1]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :D // 2], y[..., D // 2:])
    u, w = a * c - b * sn, b * c + a * sn
    out = np.empty_like(y)
    if interleaved:
        out[..., 0::2], out[..., 1::2] = u, w
    else:
        out[..., :D // 2], out[..., D // 2:] = u, w
    return out


def norm_rotate_f64(x, gain, eps, freq, pos, axis_pairs, interleaved):
    """the formulas in float64, angles from position * frequency"""
    x = np.asarray(x, np.float64)
    T, H, D = x.shape
    y = x if gain is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    ang = (pos.reshape(T, len(axis_pairs))[:, axis] * freq)[:, None]
    c, sn = np.cos(ang), np.sin(ang)
    i = np.arange(D // 2)
    fa, fb = (2 * i, 2 * i + 1) if interleaved else (i, i + D // 2)
    out = np.empty_like(y)
    out[..., fa] = y[..., fa] * c - y[..., fb] * sn
    out[..., fb] = y[..., fb] * c + y[..., fa] * sn
    return out


def rope_table(n_pos, D, axis_pairs):
    freq = np.concatenate([10000.0 ** (-np.arange(n) / max(n, 1)) for n in axis_pairs])
    ang = np.arange(n_pos, dtype=np.float64)[:, None] * freq
    return np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32), freq


def decode64(codes, meta):
    """values of FB4 codes [..., D/2] and meta [..., D/32], float64"""
    book = torch.tensor(BOOK.astype(np.float64), device=codes.device)
    m = meta.to(torch.int64)
    out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
    scale = torch.ldexp(torch.ones(m.shape, dtype=torch.float64, device=codes.device), (m & 255) - 127).repeat_interleave(16, -1)
    did = ((m >> 8) & 31).repeat_interleave(16, -1)
    for half in (0, 1):
        nib = ((codes >> (4 * half)) & 15).to(torch.int64)
        out[..., half::2] = book[did, nib & 7] * (1 - 2 * (nib >> 3)).double() * scale
    return out


def attend64(q, cache, page_table, kv_len, q_start, scale, causal, window, out_dtype):
    """(out, lse, out_tol, lse_tol) float64, rows of no sequence NaN.

    The tolerances count the roundings that the kernels make: the final one to out_dtype (half a step, relative), that of
    the probabilities to bfloat16 (2^-8 of every term of the second product), and float32 sums: a dot product of D terms is
    off by at most (D + 8) 2^-23 of its absolute sum (twice the half step: the tensor cores may truncate), which moves
    every probability by that factor, and a sum of n keys by (n + 8) 2^-23.  exp2 and the scaling add 2^-21.  The tensor-core
    kernels sum the second product times 2^-64 in float32, whose smallest step is 2^-149: each of the at most n additions can
    lose a step, 2^-85 of the result (the dividing sum is at least 1: the key that set the running maximum counts 1)."""
    total, hq, D = q.shape
    hk = cache.k_codes.shape[1]
    group = hq // hk
    page = cache.k_codes.shape[2]
    out = torch.full((total, hq, D), float("nan"), dtype=torch.float64, device=q.device)
    lse = torch.full((total, hq), float("nan"), dtype=torch.float64, device=q.device)
    otol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    step = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[out_dtype]
    n_pages = cache.k_codes.shape[0]
    for b in range(len(kv_len)):
        a0, a1, n = int(q_start[b]), int(q_start[b + 1]), int(kv_len[b])
        if a1 <= a0:
            continue
        ids = page_table[b, :-(-n // page)].long()
        ok = (ids >= 0) & (ids < n_pages)
        ids = torch.where(ok, ids, torch.zeros_like(ids))
        k = decode64(cache.k_codes[ids], cache.k_meta[ids]).transpose(0, 1).flatten(1, 2)[:, :n]
        v = decode64(cache.v_codes[ids], cache.v_meta[ids]).transpose(0, 1).flatten(1, 2)[:, :n]
        pos = n - (a1 - a0) + torch.arange(a1 - a0, device=q.device)
        j = torch.arange(n, device=q.device)
        see = ok.repeat_interleave(page)[:n][None].expand(a1 - a0, n).clone()
        if causal:
            see &= j <= pos[:, None]
        if window:
            see &= j > pos[:, None] - window
        for h in range(hq):
            qh, kh, vh = q[a0:a1, h].double(), k[h // group], v[h // group]
            z = (qh @ kh.T * scale).masked_fill(~see, float("-inf"))
            dz = (qh.abs() @ kh.abs().T * abs(scale)) * ((D + 8) * 2.0 ** -23)
            dz = dz.masked_fill(~see, 0).amax(1, keepdim=True) if n else torch.zeros(a1 - a0, 1, device=q.device, dtype=torch.float64)
            top = z.amax(1, keepdim=True) if n else torch.full((a1 - a0, 1), float("-inf"), device=q.device, dtype=torch.float64)
            top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
            p = torch.exp(z - top)
            l = p.sum(1, keepdim=True)
            w = torch.where(l > 0, p / l, torch.zeros_like(p))
            eps = 2 * dz + 2.0 ** -21 * (1 + top.abs()) + (n + 8) * 2.0 ** -23
            o, oa = w @ vh, w @ vh.abs()
            out[a0:a1, h] = o
            otol[a0:a1, h] = (2.0 ** -8 + eps) * oa * (1 + step) + step * o.abs() + n * 2.0 ** -85
            lse[a0:a1, h] = (top + torch.log(l))[:, 0]
            ltol[a0:a1, h] = (eps + 2.0 ** -22 * (1 + top.abs() + torch.log(l.clamp(min=1)).abs()))[:, 0]
    return out, lse, otol, ltol


def random_cache(q, n_pages, heads, page, D, seed, lo=119, hi=125):
    """a cache of random codes, dialects and scales"""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c = q.new_cache(n_pages, page, heads, D)
    for codes, meta in ((c.k_codes, c.k_meta), (c.v_codes, c.v_meta)):
        codes.random_(0, 256, generator=g)
        sc = torch.randint(lo, hi, meta.shape, generator=g, device="cuda")
        meta.copy_((sc | (torch.randint(0, 32, meta.shape, generator=g, device="cuda") << 8)).to(torch.int16))
    return c
