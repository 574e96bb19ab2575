"""Attention over the paged FB4 cache where numbers leave the ordinary range: scores that float32 holds only to within many powers
of two still pick the right token, in every launch shape."""
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4
from test_gpu_cache_attention import setup

pytestmark = pytest.mark.gpu

# query lengths, cache lengths, query heads, cache heads, D, page: the plain kernel; few rows in one split, in a cluster, joined by
# one and by four warps a row; many rows in one split, joined by one and by four warps a row
SHAPES = {
    "plain": ([3, 2], [70, 9], 4, 2, 96, 16),
    "few": ([1, 3], [200, 90], 8, 2, 128, 16),
    "cluster": ([1, 1], [1500, 200], 8, 2, 128, 16),
    "few, 12 splits": ([2, 1], [3000, 700], 4, 2, 64, 32),
    "few, 36 splits": ([1, 2, 1], [9000, 100, 4000], 4, 2, 128, 64),
    "many": ([40, 70], [300, 100], 8, 2, 128, 16),
    "many, 12 splits": ([150, 40], [6000, 500], 4, 2, 64, 16),
    "many, 32 splits": ([200], [20000], 1, 1, 128, 64),
}
SPLITS = {"plain": 0, "few": 0, "cluster": 0, "few, 12 splits": 12, "few, 36 splits": 36, "many": 0, "many, 12 splits": 12, "many, 32 splits": 32}


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


def in_workspace(f, name, mq, mkv):
    """splits that a call of this shape joins through its workspace"""
    q_len, _, Hq, Hk, D, _ = SHAPES[name]
    return fb4.fb4_cache_attention_workspace(f.ctx, Hq, Hk, D, len(q_len), mq, mkv, 0) / (len(q_len) * mq * Hq * (D + 2) * 4)


@pytest.mark.parametrize("q_exp,k_exp", [(8, 2), (16, 14), (45, 50)], ids=["2^16", "2^36", "2^102"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("name", SHAPES)
def test_huge_scores_pick_the_right_token(q32, name, sign, q_exp, k_exp):
    """The scores reach 2^102, where a float32 step is many powers of two of the softmax's weights.  One token stands above all
    others by more than the rounding of the scores, so it gets the whole weight."""
    q_len, kv_len, Hq, Hk, D, page = SHAPES[name]
    q, cache, table, kv, qs, mq, mkv = setup(q32, *SHAPES[name], seed=42)
    assert in_workspace(q32, name, mq, mkv) == SPLITS[name]
    scale = sign * D ** -0.5
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    base = torch.randn(Hk, D, generator=g, device="cuda")
    base = (base.sign() * base.abs().clamp(min=0.25) * 2.0 ** q_exp).to(torch.bfloat16)
    times = 2.0 ** torch.randint(0, 3, q.shape[:2], generator=g, device="cuda")
    q = (base.repeat_interleave(Hq // Hk, 0)[None].float() * times[..., None]).to(torch.bfloat16)
    cache.k_meta.copy_((cache.k_meta & ~255) | (127 + k_exp))
    want_out, want_lse = torch.zeros_like(q, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    for b in range(len(kv_len)):
        n, rows = kv_len[b], slice(int(qs[b]), int(qs[b + 1]))
        star = (n - q_len[b]) // 2                               # every query of the sequence sees it
        at = int(table[b, star // page]), slice(None), star % page
        neg = (base < 0) ^ (sign < 0)
        cache.k_codes[at] = (7 | neg[:, 0::2].to(torch.uint8) << 3 | (7 | neg[:, 1::2].to(torch.uint8) << 3) << 4)
        cache.k_meta[at] = 31 << 8 | (127 + k_exp)               # magnitude 15 in every channel, the sign of the query
        ids = table[b, :-(-n // page)].long()
        k = ref.decode64(cache.k_codes[ids], cache.k_meta[ids]).transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(Hq // Hk, 0)
        v = ref.decode64(cache.v_codes[ids], cache.v_meta[ids]).transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(Hq // Hk, 0)
        z = torch.einsum("ihd,hjd->ihj", q[rows].double(), k) * scale
        size = torch.einsum("ihd,hjd->ihj", q[rows].double().abs(), k.abs()).amax(-1) * abs(scale)
        first = z[..., star].clone()
        z[..., star] = float("-inf")
        if n > 1:                                                # a dot product is off by (D + 8) 2^-23 of its absolute sum at most
            assert (first - z.amax(-1) > 2 * (D + 8) * 2.0 ** -23 * size + 200).all()
        want_out[rows], want_lse[rows] = v[:, star][None].expand_as(want_out[rows]), first
    out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, scale=scale)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    # the weight and the result are each rounded to bfloat16: 2^-8 of the value each
    assert ((out.double() - want_out).abs() <= (2.0 ** -7 + 2.0 ** -14) * want_out.abs()).all()
    # the absolute sum of the picked token's dot product is the score itself; scaling and the factor log 2 add 2^-21
    assert ((lse.double() - want_lse).abs() <= ((D + 8) * 2.0 ** -23 + 2.0 ** -21) * want_lse.abs()).all()
