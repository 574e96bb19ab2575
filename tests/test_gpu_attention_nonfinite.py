"""Attention over the paged FB4 cache with queries that hold an infinity or NaN: NaN in every launch shape, never the zeros of a row
that sees nothing, and other rows stay right."""
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4
from test_gpu_attention_range import SHAPES
from test_gpu_cache_attention import setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("name", SHAPES)
def test_a_query_that_is_not_finite_gives_nan(q32, name, what):
    q_len, kv_len, Hq, Hk, D, page = SHAPES[name]
    q, cache, table, kv, qs, mq, mkv = setup(q32, *SHAPES[name], seed=40)
    want = ref.attend64(q, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16)
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for row, head in {(0, 0), (q.shape[0] - 1, Hq - 1), (q.shape[0] // 2, Hq // 2)}:
        q[row, head, (7 * row + 3) % D] = what                   # one channel; the last one of them in all channels
        hit[row, head] = True
    q[-1, -1] = what
    out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert ((out.double() - want[0]).abs() <= want[2])[~hit].all() and ((lse.double() - want[1]).abs() <= want[3])[~hit].all()


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("n_q", [4, 90])
def test_a_query_that_sees_nothing_gives_zeros_whatever_it_holds(q32, n_q, D):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [n_q, n_q], [n_q - 2, 0], 4, 2, D, 16, seed=41)
    q[0, 1], q[1, 0, 3], q[n_q + 1, 2] = float("nan"), float("inf"), float("-inf")
    out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    for empty in (slice(0, 2), slice(n_q, 2 * n_q)):
        assert not out[empty].any() and (lse[empty] == float("-inf")).all()
    assert torch.isfinite(out[2:n_q].float()).all()


@pytest.mark.parametrize("name", SHAPES)
def test_scores_beyond_float32(q32, name):
    """upwards: NaN; downwards: no weight, so the one token whose score is zero takes all of it"""
    q_len, kv_len, Hq, Hk, D, page = SHAPES[name]
    q, cache, table, kv, qs, mq, mkv = setup(q32, *SHAPES[name], seed=43)
    q = (q.abs().float().clamp(min=1) * 2.0 ** 100).to(torch.bfloat16)
    cache.k_codes.copy_(cache.k_codes & 0x77 | 0x11)               # every key positive, and none zero
    cache.k_meta.copy_((cache.k_meta & ~255) | 180)
    out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, scale=2.0 ** 60)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    want = torch.empty_like(q)
    for b, n in enumerate(kv_len):
        star = (n - q_len[b]) // 2                                 # every query of the sequence sees it
        cache.k_codes[int(table[b, star // page]), :, star % page] = 0
        ids = table[b, :-(-n // page)].long()
        v = ref.decode64(cache.v_codes[ids], cache.v_meta[ids]).transpose(1, 2).flatten(0, 1)[star].repeat_interleave(Hq // Hk, 0)
        want[int(qs[b]):int(qs[b + 1])] = v.to(torch.bfloat16)     # an FB4 value is a bfloat16 number
    out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, scale=-2.0 ** 60)
    assert torch.equal(out, want) and not lse.any()


@pytest.mark.parametrize("name", SHAPES)
def test_subnormal_queries_count(q32, name):
    q_len, kv_len, Hq, Hk, D, page = SHAPES[name]
    q, cache, table, kv, qs, mq, mkv = setup(q32, *SHAPES[name], seed=44)
    q = (q.float() * 2.0 ** -130).to(torch.bfloat16)
    assert q.any() and q.abs().max() < 2.0 ** -126
    cache.k_meta.copy_((cache.k_meta & ~255) | 187)                # element scale 2^60
    scale = 2.0 ** 60
    want = ref.attend64(q, cache, table, kv, qs, scale, True, 0, torch.bfloat16)
    flat = ref.attend64(q * 0, cache, table, kv, qs, scale, True, 0, torch.bfloat16)
    assert ((want[1] - flat[1]).abs() > 2 * want[3]).any()         # they do move the result
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, scale=scale)
    assert ((got[0].double() - want[0]).abs() <= want[2]).all() and ((got[1].double() - want[1]).abs() <= want[3]).all()
