"""Attention over the paged FB4 cache against float64: lengths from none to long, groups, masks that leave rows empty, pages
that end inside a tile, bad pages, strided queries, output types; a layer's run of append and attention; refusals."""
import numpy as np
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def setup(f, q_len, kv_len, Hq, Hk, D, page, seed=0, spread=1.5):
    q_len, kv_len = np.asarray(q_len), np.asarray(kv_len)
    need = -(-kv_len // page)
    n_pages = int(need.sum()) + 2
    rng = np.random.default_rng(seed)
    perm = rng.permutation(n_pages)
    table = np.full((len(kv_len), max(1, int(need.max()))), -7, np.int32)          # entries behind the last page are never read
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = (torch.randn(int(q_len.sum()), Hq, D, generator=g, device="cuda") * spread).to(torch.bfloat16)
    cache = ref.random_cache(f, n_pages, Hk, page, D, seed)
    return q, cache, i32(table), i32(kv_len), i32(np.concatenate([[0], np.cumsum(q_len)])), int(q_len.max()), int(kv_len.max())


def agree(got, want, dtype=torch.bfloat16):
    out, lse = got
    o, l, otol, ltol = want
    rows = ~torch.isnan(o[:, 0, 0])
    d = (out.double() - o).abs()[rows]
    assert torch.isfinite(out[rows].float()).all()
    assert (d <= otol[rows] + 1e-30).all(), f"out off by {float((d / (otol[rows] + 1e-30)).max()):.3g} of what is allowed"
    inf = torch.isinf(l) & rows[:, None]
    assert torch.equal(torch.isinf(lse) & rows[:, None], inf) and (lse[inf] < 0).all()
    ok = rows[:, None] & ~inf
    assert ((lse.double() - l).abs()[ok] <= ltol[ok]).all()


CASES = [
    # q lengths, cache lengths, query heads, cache heads, D, page
    ([1], [1], 1, 1, 128, 16), ([1], [17], 8, 8, 128, 16), ([1], [1023], 8, 2, 64, 32), ([1, 1, 1], [1, 300, 64], 32, 8, 128, 16),
    ([1], [5000], 12, 12, 128, 64), ([1] * 9, [0, 1, 15, 16, 17, 127, 128, 129, 1000], 6, 2, 64, 16),
    ([2, 3, 1], [2, 200, 33], 16, 4, 128, 16), ([5], [5], 7, 1, 64, 16), ([6, 2], [700, 90], 16, 1, 128, 4096), ([3], [40], 5, 5, 96, 16),
    ([4, 0, 2], [100, 50, 7], 4, 2, 32, 32), ([2], [65], 3, 1, 256, 128), ([17], [1000], 8, 2, 128, 32), ([100, 1, 40], [100, 513, 40], 4, 2, 64, 16),
    ([129], [257], 4, 4, 128, 64), ([200, 300], [200, 900], 8, 1, 128, 16), ([512], [1000], 3, 3, 64, 128), ([33, 64, 128], [640, 64, 500], 12, 4, 128, 16),
]


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 37), (False, 1)])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}-{c[1]}-{c[2]}.{c[3]}.{c[4]}.{c[5]}".replace(" ", "") for c in CASES])
def test_matches_float64(q32, case, causal, window):
    q, cache, table, kv, qs, mq, mkv = setup(q32, *case, seed=len(str(case)))
    D = case[4]
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window)
    agree(got, ref.attend64(q, cache, table, kv, qs, D ** -0.5, causal, window, torch.bfloat16))
    assert q32.device_status == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("n_q", [1, 80])
def test_output_types(q32, dtype, n_q):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [n_q, 2], [300, 33], 8, 2, 128, 16, seed=4)
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, scale=0.03, dtype=dtype)
    assert got[0].dtype == dtype
    agree(got, ref.attend64(q, cache, table, kv, qs, 0.03, True, 0, dtype))


@pytest.mark.parametrize("n_q,D", [(1, 128), (3, 64), (150, 128), (150, 64)])
def test_rows_that_see_nothing(q32, n_q, D):
    """more queries than cached tokens: the first ones stand before the cache begins"""
    q, cache, table, kv, qs, mq, mkv = setup(q32, [n_q + 2, n_q], [n_q, 0], 4, 2, D, 16, seed=3)
    out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    assert not out[:2].any() and torch.isinf(lse[:2]).all() and not out[n_q + 2:].any() and torch.isinf(lse[n_q + 2:]).all()
    agree((out, lse), ref.attend64(q, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16))


@pytest.mark.parametrize("n_q", [1, 70])
def test_extreme_scores_and_values(q32, n_q):
    """scores of thousands (one key takes all) and values near the largest and smallest that the format holds"""
    q, cache, table, kv, qs, mq, mkv = setup(q32, [n_q], [300], 4, 2, 128, 16, seed=6, spread=200.0)
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, scale=1.0)
    agree(got, ref.attend64(q, cache, table, kv, qs, 1.0, True, 0, torch.bfloat16))
    q = q / 200
    cache.v_meta.copy_((cache.v_meta & ~255) | 188)            # element scale 2^61
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    agree(got, ref.attend64(q, cache, table, kv, qs, 128 ** -0.5, True, 0, torch.bfloat16))
    cache.v_meta.copy_((cache.v_meta & ~255) | 59)             # 2^-68
    cache.k_meta.copy_((cache.k_meta & ~255) | 1)              # keys that are all but zero
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, dtype=torch.float32)
    agree(got, ref.attend64(q, cache, table, kv, qs, 128 ** -0.5, True, 0, torch.float32))


@pytest.mark.parametrize("n_q", [1, 70])
def test_scales_beyond_the_readable_range_count_as_its_end(q32, n_q):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [n_q], [130], 2, 2, 64, 16, seed=6)
    cache.v_meta.copy_((cache.v_meta & ~255) | 188)
    want = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, dtype=torch.float32)
    cache.v_meta.copy_((cache.v_meta & ~255) | 251)
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, dtype=torch.float32)
    assert torch.equal(got[0], want[0])


@pytest.mark.parametrize("n_q", [1, 90])
@pytest.mark.parametrize("D", [64, 128])
def test_what_lies_behind_the_last_token_does_not_matter(q32, n_q, D):
    """slots of the last page behind kv_len hold any bytes: scales that decode to infinity, dialect bits that are none"""
    q, cache, table, kv, qs, mq, mkv = setup(q32, [n_q], [203], 4, 2, D, 32, seed=8)
    want = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    page = int(table[0, 203 // 32])
    for t in (cache.k_meta, cache.v_meta):
        t[page, :, 203 % 32:] = -1
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n_q,Hq", [(1, 4), (5, 8), (100, 4)])
def test_a_bad_page_is_left_out_and_reported(n_q, Hq):
    f = fb4.Fb4()
    q, cache, table, kv, qs, mq, mkv = setup(f, [n_q, n_q], [400, 300], Hq, 2, 128, 32, seed=9)
    table[0, 3], table[1, 0] = cache.k_codes.shape[0], -1
    got = f.cache_attention(q, cache, table, kv, qs, mq, mkv)
    agree(got, ref.attend64(q, cache, table, kv, qs, 128 ** -0.5, True, 0, torch.bfloat16))
    assert f.device_status == 2
    f.close()


def test_lengths_outside_their_bounds_are_clamped_and_reported():
    f = fb4.Fb4()
    q, cache, table, kv, qs, mq, mkv = setup(f, [2, 3], [100, 60], 2, 2, 64, 16, seed=2)
    bad_kv, bad_qs = kv.clone(), qs.clone()
    bad_kv[0], bad_qs[2] = 10 ** 6, 400
    got = f.cache_attention(q, cache, table, bad_kv, bad_qs, mq, mkv)
    want = f.cache_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(got[0], want[0]) and f.device_status == 2
    f.close()


def test_strided_queries_and_rows_of_no_sequence(q32):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [3, 60], [90, 100], 4, 2, 128, 16, seed=12)
    big = torch.zeros(70, 10, 128, dtype=torch.bfloat16, device="cuda")
    big[:63, 2:6] = q
    out = torch.full((70, 6 * 128), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((70, 4), 5.0, device="cuda")
    need = fb4.fb4_cache_attention_workspace(q32.ctx, 4, 2, 128, 2, mq, mkv, 0)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    fb4.fb4_cache_attention(q32.ctx, big[:, 2:], 1280, 4, 70, q32._cache(cache), table, table.shape[1], kv, qs, 2, mq, mkv, 128 ** -0.5,
                            True, 0, out[:, 128:], 768, 1, lse, ws if need else None, need)
    want = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(out[:63, 128:640].reshape(63, 4, 128), want[0]) and torch.equal(lse[:63], want[1])
    assert (out[63:] == 5).all() and (out[:, :128] == 5).all() and (out[:, 640:] == 5).all() and (lse[63:] == 5).all()


def test_the_plain_kernel_agrees(q32):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [1, 40], [333, 80], 8, 2, 128, 16, seed=13)
    q32.set_kernel_variant(1)
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, window=50)
    assert q32.last_variant == "generic"
    q32.set_kernel_variant(0)
    agree(got, ref.attend64(q, cache, table, kv, qs, 128 ** -0.5, True, 50, torch.bfloat16))


def test_a_layer_step_by_step_equals_the_whole_prompt(q32):
    """append + attention of a prompt at once, in two chunks, and token by token, on a stream of their own: the cache is the same
    bit for bit, and every form agrees with float64"""
    T, Hq, Hk, D, page = 50, 8, 2, 128, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(T, Hq + 2 * Hk, D, generator=g, device="cuda").to(torch.bfloat16)
    gains = (1 + 0.1 * torch.randn(2, D, generator=g, device="cuda")).to(torch.bfloat16)
    tab = torch.from_numpy(ref.rope_table(64, D, (64,))[0]).cuda()
    table = i32([[2, 0, 3, 1]])

    def run(steps):
        cache = q32.new_cache(4, page, Hk, D)
        outs, at = [], 0
        for n in steps:
            pos = torch.arange(at, at + n, device="cuda")
            slot = table[0].long()[pos // page] * page + pos % page
            xs = x[at:at + n]
            qo = q32.cache_append(cache, slot, xs[:, Hq:Hq + Hk], xs[:, Hq + Hk:], gains[1], 1e-6, fb4.Rope(tab, pos.int(), [64]),
                                  q=xs[:, :Hq], q_gain=gains[0])
            at += n
            out, lse = q32.cache_attention(qo, cache, table, i32([at]), i32([0, n]), n, at)
            outs.append((qo, out, lse))
        return cache, [torch.cat(t) for t in zip(*outs)]
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        runs = [run(s) for s in ([T], [33, 17], [1] * T)]
    st.synchronize()
    whole = ref.attend64(runs[0][1][0], runs[0][0], table, i32([T]), i32([0, T]), D ** -0.5, True, 0, torch.bfloat16)
    for cache, (qo, out, lse) in runs:
        assert torch.equal(cache.k_codes, runs[0][0].k_codes) and torch.equal(cache.v_meta, runs[0][0].v_meta) and torch.equal(qo, runs[0][1][0])
        agree((out, lse), whole)


@pytest.mark.parametrize("q_len,kv_len,heads", [([1, 1], [1500, 200], (8, 2)), ([1, 1], [30000, 20000], (2, 1)), ([150, 40], [6000, 500], (2, 1))],
                         ids=["cluster", "few rows, workspace", "many rows, workspace"])
def test_captured_and_replayed(q32, q_len, kv_len, heads):
    q, cache, table, kv, qs, mq, mkv = setup(q32, q_len, kv_len, *heads, 128, 16, seed=14)
    assert (fb4.fb4_cache_attention_workspace(q32.ctx, *heads, 128, 2, mq, mkv, 0) > 0) == (mkv > 3000)
    want = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=st):
        got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    for _ in range(3):
        got[0].zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q2 = torch.randn_like(q)
    kv2 = kv // 2 + 75
    want = q32.cache_attention(q2, cache, table, kv2, qs, mq, mkv)
    q.copy_(q2)
    kv.copy_(kv2)
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0])


def test_two_calls_at_once_on_two_streams(q32):
    """every call has a workspace of its own; contexts are only serialised on the host"""
    args = [setup(q32, [1, 2], [20000, 9000], 4, 1, 128, 16, seed=20), setup(q32, [100, 60], [4000, 9000], 2, 2, 64, 32, seed=21)]
    want = [q32.cache_attention(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(8):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(q32.cache_attention(*args[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert torch.equal(g[0], want[i][0]) and torch.equal(g[1], want[i][1])


@pytest.mark.parametrize("n_q", [1, 40])
def test_a_cache_whose_offsets_pass_32_bits(q32, n_q):
    """4.6 GB of codes for K and for V; the sequence lives in the last pages and in the first"""
    heads, page, D = 8, 64, 128
    n_pages = (1 << 32) // (heads * page * D // 2) + 16000
    codes = [torch.empty(n_pages, heads, page, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    meta = [torch.empty(n_pages, heads, page, D // 32, dtype=torch.int16, device="cuda") for _ in range(2)]
    big = fb4.Cache(codes[0], meta[0], codes[1], meta[1])
    ids = [n_pages - 1, 0, n_pages - 7, 131072, 3]
    n = 5 * page - 9
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    kv = torch.randn(2, n, heads, D, generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn(n_q, heads, D, generator=g, device="cuda").to(torch.bfloat16)
    at = torch.arange(n, device="cuda")
    slot = torch.tensor(ids, device="cuda")[at // page] * page + at % page
    assert int(slot.max()) * heads * D // 2 > 1 << 32
    small = q32.new_cache(5, page, heads, D)
    q32.cache_append(big, slot, kv[0], kv[1])
    q32.cache_append(small, at, kv[0], kv[1])
    a = q32.cache_attention(q, big, i32([ids]), i32([n]), i32([0, n_q]), n_q, n)
    b = q32.cache_attention(q, small, i32([[0, 1, 2, 3, 4]]), i32([n]), i32([0, n_q]), n_q, n)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(big.k_codes[ids[0]], small.k_codes[0]) and torch.equal(big.v_meta[ids[3]], small.v_meta[3])


def test_refusals(q32):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [2, 3], [100, 60], 4, 2, 64, 16, seed=2)
    c = q32._cache(cache)
    out = torch.empty(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    need = fb4.fb4_cache_attention_workspace(q32.ctx, 4, 2, 64, 2, mq, mkv, 0)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    ok = dict(q=q, q_ld=256, q_heads=4, total_q=5, cache=c, page_table=table, max_pages=table.shape[1], kv_len=kv, q_start=qs, n_seqs=2,
              max_q=mq, max_kv=mkv, scale=0.1, causal=True, window=0, out=out, out_ld=256, out_dtype=1, lse=None, workspace=ws,
              workspace_bytes=ws.numel())

    def code(ctx=q32.ctx, **change):
        try:
            fb4.fb4_cache_attention(ctx, **{**ok, **change})
        except fb4.Fb4Error as e:
            return e.code
        return 0
    assert code() == 0 and code(total_q=0) == 0 and code(n_seqs=0) == 0 and code(max_q=0) == 0
    assert code(q_heads=3) == fb4.ERR_SHAPE and code(q_heads=0) == fb4.ERR_SHAPE and code(n_seqs=-1) == fb4.ERR_SHAPE
    assert code(max_kv=-1) == fb4.ERR_SHAPE and code(q_ld=200) == fb4.ERR_SHAPE and code(out_ld=128) == fb4.ERR_SHAPE
    assert code(window=-1) == fb4.ERR_INVALID_ARG and code(out_dtype=3) == fb4.ERR_INVALID_ARG and code(scale=float("nan")) == fb4.ERR_INVALID_ARG
    assert code(scale=float("inf")) == fb4.ERR_INVALID_ARG and code(kv_len=None) == fb4.ERR_INVALID_ARG and code(q=None) == fb4.ERR_INVALID_ARG
    assert code(page_table=None) == fb4.ERR_INVALID_ARG and code(out=None) == fb4.ERR_INVALID_ARG
    assert code(q=q.data_ptr() + 2) == fb4.ERR_ALIGN and code(out=out.data_ptr() + 8) == fb4.ERR_ALIGN and code(out_ld=260) == fb4.ERR_ALIGN
    assert code(workspace=ws.data_ptr() + 16) == fb4.ERR_ALIGN and code(kv_len=kv.data_ptr() + 2) == fb4.ERR_ALIGN
    if need:
        assert code(workspace=None) == fb4.ERR_INVALID_ARG and code(workspace_bytes=need - 1) == fb4.ERR_INVALID_ARG
    assert fb4.fb4_cache_attention_workspace(q32.ctx, 3, 2, 64, 1, 1, 1, 0) == -1
    z = fb4.Fb4(block_size=16)
    assert code(ctx=z.ctx) == fb4.ERR_INVALID_ARG
    z.close()
    with pytest.raises(ValueError):
        q32.cache_attention(q, cache, table, kv.long(), qs, mq, mkv)
    with pytest.raises(ValueError):
        q32.cache_attention(q[..., :32], cache, table, kv, qs, mq, mkv)


def test_sizes_that_do_not_fit_32_bits_are_refused(q32):
    q, cache, table, kv, qs, mq, mkv = setup(q32, [2], [100], 4, 2, 64, 16, seed=2)
    for bad in ((2 ** 32 + mq, mkv, 0), (mq, 2 ** 32 + mkv, 0), (mq, mkv, 2 ** 32 + 1), (mq, mkv, 2 ** 63 - 1), (mq, mkv, -1)):
        with pytest.raises(ValueError):
            q32.cache_attention(q, cache, table, kv, qs, *bad[:2], window=bad[2])
    want = q32.cache_attention(q, cache, table, kv, qs, mq, mkv)
    got = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, window=2 ** 31 - 1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and q32.last_variant == "fast"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_row_tiles_that_see_nothing(q32, D, dtype):
    """whole tiles of query rows stand before the cache begins: they have no tile of tokens to wait for, and still get zeros"""
    q, cache, table, kv, qs, mq, mkv = setup(q32, [18, 33, 7] * 20, [2, 1, 60] * 20, 128, 8, D, 128, seed=30)
    want = ref.attend64(q[:58], cache, table[:3], kv[:3], qs[:4], D ** -0.5, True, 0, dtype)
    for _ in range(5):
        out, lse = q32.cache_attention(q, cache, table, kv, qs, mq, mkv, dtype=dtype)
        agree((out[:58], lse[:58]), want, dtype)
        o, l = out.view(20, 58, 128, D), lse.view(20, 58, 128)
        empty = torch.cat([torch.arange(16), 18 + torch.arange(32)]).cuda()
        assert not o[:, empty].any() and torch.isinf(l[:, empty]).all()


@pytest.mark.parametrize("case", [([1, 3], 4, 16), ([70, 5], 4, 32), ([300, 150], 2, 64)], ids=["few", "many", "several tiles"])
@pytest.mark.parametrize("D", [64, 128])
def test_pages_in_front_of_the_window_may_be_gone(case, D):
    """a page that no query sees is neither read nor reported, also where tiles of tokens begin in front of the window"""
    n_q, group, page = case
    f = fb4.Fb4()
    q, cache, table, kv, qs, mq, mkv = setup(f, n_q, [1000, 777], 2 * group, 2, D, page, seed=31)
    want = f.cache_attention(q, cache, table, kv, qs, mq, mkv, window=100)
    for b, (n, k) in enumerate(zip([1000, 777], n_q)):
        table[b, :(n - k - 100 + 1) // page] = -1
    got = f.cache_attention(q, cache, table, kv, qs, mq, mkv, window=100)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and f.device_status == 0
    f.close()
