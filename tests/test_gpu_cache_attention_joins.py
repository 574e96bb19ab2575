"""Attention over the paged FB4 cache where the cached tokens are split over CTAs and joined through the workspace, against
float64: both kernels, both forms of the join, causal and not, windows, lengths that leave splits empty, all output types; bounds far above
the real lengths; head dimensions of the plain kernel over longer caches; guard bytes around the workspace and the outputs;
refusals of a workspace that is missing or short."""
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4
from test_gpu_cache_attention import agree, setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


def joined(f, shape, mq, mkv, window):
    """splits that a call of this shape joins through its workspace, 0 = none"""
    q_len, _, Hq, Hk, D, _ = shape
    need = fb4.fb4_cache_attention_workspace(f.ctx, Hq, Hk, D, len(q_len), mq, mkv, window)
    per = len(q_len) * mq * Hq * (D + 2) * 4
    assert need % per == 0
    return need // per


# query lengths, cache lengths, query heads, cache heads, D, page; causal, window, splits
CASES = [
    (([1, 1], [3000, 700], 8, 2, 128, 16), True, 0, 12), (([2, 1, 2], [3000, 0, 41], 4, 2, 64, 32), False, 0, 12),
    (([6, 1], [2900, 1024], 4, 2, 128, 64), True, 0, 12), (([3, 2], [9000, 5000], 8, 2, 64, 128), True, 2500, 10),
    (([1, 1, 1], [9000, 100, 4000], 4, 2, 64, 16), True, 0, 36), (([1, 2, 1], [9000, 3, 2048], 4, 2, 128, 64), False, 0, 36),
    (([7, 3], [9001, 4500], 4, 2, 64, 32), True, 0, 36), (([15], [9000], 2, 1, 128, 16), False, 6000, 24),
    (([5, 1], [12000, 33], 2, 2, 128, 4096), True, 6001, 24),
    (([150, 40, 1], [6000, 500, 40], 4, 2, 64, 16), True, 0, 12), (([150, 40], [6000, 500], 4, 2, 128, 64), False, 0, 12),
    (([130, 129], [7000, 6900], 4, 2, 128, 32), True, 2000, 0), (([260, 100], [6000, 5000], 2, 2, 64, 128), False, 2000, 0),
    (([200], [20000], 1, 1, 128, 64), True, 0, 32), (([100], [20011], 2, 1, 64, 16), False, 0, 32), (([700], [9000], 1, 1, 64, 64), True, 0, 0),
    (([300], [250], 1, 1, 128, 16), True, 0, 0),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16])
@pytest.mark.parametrize("case", CASES, ids=[f"{s}-{c}-{w}-{n}".replace(" ", "") for s, c, w, n in CASES])
def test_joined_splits_match_float64(q32, case, dtype):
    shape, causal, window, splits = case
    D = shape[4]
    q, cache, table, kv, qs, mq, mkv = setup(q32, *shape, seed=50)
    n = joined(q32, shape, mq, mkv, window)
    assert n == splits if splits else n == 0 or n > 1
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window, dtype=dtype)
    agree(got, ref.attend64(q, cache, table, kv, qs, D ** -0.5, causal, window, dtype), dtype)
    again = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window, dtype=dtype)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1]) and q32.device_status == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,max_q,max_kv", [([1, 2], 2, 60000), ([1, 1], 12, 20000), ([60, 33], 64, 50000), ([60, 3], 300, 9000), ([2, 1], 40, 9000)])
def test_bounds_far_above_the_lengths(q32, n_q, max_q, max_kv, D):
    """a captured step has the largest lengths as its bounds: most splits are then empty, or all but the first"""
    q, cache, table, kv, qs, _, _ = setup(q32, n_q, [130, 1000], 4, 2, D, 32, seed=51)
    got = q32.cache_attention(q, cache, table, kv, qs, max_q, max_kv)
    agree(got, ref.attend64(q, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16))
    assert q32.device_status == 0


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 300)])
@pytest.mark.parametrize("shape", [([1, 1], [2500, 900], 4, 2, 96, 16), ([5, 40], [1300, 700], 8, 2, 96, 64), ([1, 3], [1800, 31], 4, 4, 256, 32),
                                   ([33], [1025], 2, 1, 256, 128), ([9, 2], [600, 1500], 4, 2, 32, 16), ([4], [1111], 3, 1, 192, 16)])
def test_head_dimensions_of_the_plain_kernel(q32, shape, causal, window):
    D = shape[4]
    q, cache, table, kv, qs, mq, mkv = setup(q32, *shape, seed=52)
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window, dtype=torch.float32)
    agree(got, ref.attend64(q, cache, table, kv, qs, D ** -0.5, causal, window, torch.float32))


@pytest.mark.parametrize("shape", [([1, 3], [9000, 400], 4, 2, 64, 16), ([5], [12000], 2, 1, 128, 64), ([150, 3], [6000, 500], 4, 2, 64, 16),
                                   ([130], [9000], 3, 1, 128, 32), ([1, 1], [1500, 200], 8, 2, 128, 16), ([3], [50], 2, 1, 96, 16)])
def test_nothing_is_written_outside_the_workspace_and_the_outputs(q32, shape):
    """guard bytes on both sides of each, the workspace exactly as large as asked for"""
    q_len, _, Hq, Hk, D, _ = shape
    q, cache, table, kv, qs, mq, mkv = setup(q32, *shape, seed=53)
    total, n = q.shape[0], len(q_len)
    want = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    held = [t.clone() for t in (cache.k_codes, cache.k_meta, cache.v_codes, cache.v_meta)]
    need = fb4.fb4_cache_attention_workspace(q32.ctx, Hq, Hk, D, n, mq, mkv, 0)
    sizes = [total * Hq * D * 2, total * Hq * 4, need]
    raw = [torch.full((4096 + -(-s // 256) * 256 + 4096,), 0xA5, dtype=torch.uint8, device="cuda") for s in sizes]
    at = [r[4096:4096 + s] for r, s in zip(raw, sizes)]
    fb4.fb4_cache_attention(q32.ctx, q, Hq * D, Hq, total, q32._cache(cache), table, table.shape[1], kv, qs, n, mq, mkv, D ** -0.5, True, 0,
                            at[0], Hq * D, 1, at[1], at[2] if need else None, need)
    torch.cuda.synchronize()
    for r, s in zip(raw, sizes):
        assert (r[:4096] == 0xA5).all() and (r[4096 + s:] == 0xA5).all()
    assert torch.equal(at[0].view(torch.bfloat16).view(total, Hq, D), want[0]) and torch.equal(at[1].view(torch.float32).view(total, Hq), want[1])
    for a, b in zip(held, (cache.k_codes, cache.k_meta, cache.v_codes, cache.v_meta)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [([1, 1], [20000, 40], 4, 2, 64, 16), ([150, 2], [6000, 70], 4, 2, 128, 16)])
def test_a_workspace_that_is_missing_or_short_is_refused(q32, shape):
    q_len, _, Hq, Hk, D, _ = shape
    q, cache, table, kv, qs, mq, mkv = setup(q32, *shape, seed=54)
    need = fb4.fb4_cache_attention_workspace(q32.ctx, Hq, Hk, D, 2, mq, mkv, 0)
    assert need > 0
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def code(workspace, size):
        try:
            fb4.fb4_cache_attention(q32.ctx, q, Hq * D, Hq, q.shape[0], q32._cache(cache), table, table.shape[1], kv, qs, 2, mq, mkv, 0.1, True,
                                    0, out, Hq * D, 1, None, workspace, size)
        except fb4.Fb4Error as e:
            return e.code
        return 0
    before = q32.launch_count
    assert code(None, need) == fb4.ERR_INVALID_ARG and code(ws, need - 1) == fb4.ERR_INVALID_ARG and code(ws, 0) == fb4.ERR_INVALID_ARG
    assert code(ws, -1) == fb4.ERR_INVALID_ARG and q32.launch_count == before
    assert code(ws, need) == 0 and q32.launch_count == before + 2
