"""Attention over the paged 8-bit cache against float64: lengths from none to long, groups, masks that leave rows empty, pages that end
inside a tile, splits, bad pages, strided queries, output types, numbers out of the ordinary range; a server's steps of plan, append and
attention; refusals."""
import pytest
import torch

import attend_ref
import cache8_ref as ref
from paper_2603_02883_b200 import fb4
from test_gpu_attention_range import SHAPES
from test_gpu_cache_attention import CASES, agree
from test_gpu_cache_attention_joins import CASES as JOINS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def f():
    q = fb4.Fb4()
    yield q
    q.close()


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 37), (False, 1)])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}-{c[1]}-{c[2]}.{c[3]}.{c[4]}.{c[5]}".replace(" ", "") for c in CASES])
def test_matches_float64(f, case, causal, window):
    q, cache, table, kv, qs, mq, mkv = ref.setup(*case, seed=len(str(case)))
    D = case[4]
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window)
    agree(got, ref.attend64(q, cache, table, kv, qs, D ** -0.5, causal, window, torch.bfloat16))
    assert f.device_status == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16])
@pytest.mark.parametrize("case", JOINS, ids=[f"{s}-{c}-{w}".replace(" ", "") for s, c, w, n in JOINS])
def test_longer_caches_match_float64(f, case, dtype):
    shape, causal, window, _ = case
    q, cache, table, kv, qs, mq, mkv = ref.setup(*shape, seed=50)
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window, dtype=dtype)
    agree(got, ref.attend64(q, cache, table, kv, qs, shape[4] ** -0.5, causal, window, dtype), dtype)
    again = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, causal=causal, window=window, dtype=dtype)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1]) and f.device_status == 0


@pytest.mark.parametrize("n_q,D", [(1, 128), (3, 64), (150, 128), (150, 64), (2, 96)])
def test_rows_that_see_nothing(f, n_q, D):
    q, cache, table, kv, qs, mq, mkv = ref.setup([n_q + 2, n_q], [n_q, 0], 4, 2, D, 16, seed=3)
    out, lse = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    assert not out[:2].any() and torch.isinf(lse[:2]).all() and not out[n_q + 2:].any() and torch.isinf(lse[n_q + 2:]).all()
    agree((out, lse), ref.attend64(q, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16))


@pytest.mark.parametrize("scales", [(58, 59), (185, 186), (58, 186)], ids=["smallest", "largest", "both"])
@pytest.mark.parametrize("name", SHAPES)
def test_the_ends_of_the_scales(f, name, scales):
    """every value is read exactly, down to 2^-69 and up to 127 * 2^58, also side by side"""
    q, cache, table, kv, qs, mq, mkv = ref.setup(*SHAPES[name], seed=6)
    D = SHAPES[name][4]
    rand = torch.randint(*scales, cache.v_scale.shape, device="cuda", dtype=torch.uint8)
    cache.v_scale.copy_(torch.where(rand > 120, 185, 58) if scales == (58, 186) else rand)
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, dtype=torch.float32)
    agree(got, ref.attend64(q, cache, table, kv, qs, D ** -0.5, True, 0, torch.float32), torch.float32)
    want, kept = got, cache.v_scale.clone()
    cache.v_scale[kept == 185] = 251                          # out of range: read as the nearest that is in it
    cache.v_scale[kept == 58] = 3
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, dtype=torch.float32)
    assert torch.equal(got[0], want[0])
    cache.v_scale.fill_(120)
    cache.k_scale.fill_(185)
    small = (q.float() * 2.0 ** -60).to(torch.bfloat16)
    got = f.cache8_attention(small, cache, table, kv, qs, mq, mkv)
    agree(got, ref.attend64(small, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16))
    cache.k_scale.fill_(58)
    small = (q.float() * 2.0 ** 62).to(torch.bfloat16)
    got = f.cache8_attention(small, cache, table, kv, qs, mq, mkv)
    agree(got, ref.attend64(small, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16))


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("name", SHAPES)
def test_peaked_rows(f, name, sign):
    """scores of thousands, and a scale below zero"""
    q, cache, table, kv, qs, mq, mkv = ref.setup(*SHAPES[name], seed=7, spread=100.0)
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, scale=0.2 * sign)
    agree(got, ref.attend64(q, cache, table, kv, qs, 0.2 * sign, True, 0, torch.bfloat16))


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("name", SHAPES)
def test_a_query_that_is_not_finite_gives_nan(f, name, what):
    q, cache, table, kv, qs, mq, mkv = ref.setup(*SHAPES[name], seed=40)
    D, Hq = SHAPES[name][4], SHAPES[name][2]
    want = ref.attend64(q, cache, table, kv, qs, D ** -0.5, True, 0, torch.bfloat16)
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for row, head in {(0, 0), (q.shape[0] - 1, Hq - 1), (q.shape[0] // 2, Hq // 2)}:
        q[row, head, (7 * row + 3) % D] = what
        hit[row, head] = True
    out, lse = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert ((out.double() - want[0]).abs() <= want[2])[~hit].all() and ((lse.double() - want[1]).abs() <= want[3])[~hit].all()


@pytest.mark.parametrize("n_q", [1, 90])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_what_lies_behind_the_last_token_does_not_matter(f, n_q, D):
    q, cache, table, kv, qs, mq, mkv = ref.setup([n_q], [203], 4, 2, D, 32, seed=8)
    want = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    page = int(table[0, 203 // 32])
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        t[page, :, 203 % 32:] = 0
        s[page, :, 1:] = 255
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n_q,Hq", [(1, 4), (5, 8), (100, 4)])
def test_a_bad_page_is_left_out_and_reported(n_q, Hq):
    f = fb4.Fb4()
    q, cache, table, kv, qs, mq, mkv = ref.setup([n_q, n_q], [400, 300], Hq, 2, 128, 32, seed=9)
    table[0, 3], table[1, 0] = cache.k.shape[0], -1
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    agree(got, ref.attend64(q, cache, table, kv, qs, 128 ** -0.5, True, 0, torch.bfloat16))
    assert f.device_status == 2
    f.close()


def test_lengths_outside_their_bounds_are_clamped_and_reported():
    f = fb4.Fb4()
    q, cache, table, kv, qs, mq, mkv = ref.setup([2, 3], [100, 60], 2, 2, 64, 16, seed=2)
    bad_kv, bad_qs = kv.clone(), qs.clone()
    bad_kv[0], bad_qs[2] = 10 ** 6, 400
    got = f.cache8_attention(q, cache, table, bad_kv, bad_qs, mq, mkv)
    want = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(got[0], want[0]) and f.device_status == 2
    f.close()


@pytest.mark.parametrize("case", [([1, 3], 4, 16), ([70, 5], 4, 32), ([300, 150], 2, 64)], ids=["few", "many", "several tiles"])
@pytest.mark.parametrize("D", [64, 128])
def test_pages_in_front_of_the_window_may_be_gone(case, D):
    n_q, group, page = case
    f = fb4.Fb4()
    q, cache, table, kv, qs, mq, mkv = ref.setup(n_q, [1000, 777], 2 * group, 2, D, page, seed=31)
    want = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, window=100)
    for b, (n, k) in enumerate(zip([1000, 777], n_q)):
        table[b, :(n - k - 100 + 1) // page] = -1
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, window=100)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and f.device_status == 0
    f.close()


def test_strided_queries_and_rows_of_no_sequence(f):
    q, cache, table, kv, qs, mq, mkv = ref.setup([3, 60], [90, 100], 4, 2, 128, 16, seed=12)
    big = torch.zeros(70, 10, 128, dtype=torch.bfloat16, device="cuda")
    big[:63, 2:6] = q
    out = torch.full((70, 6 * 128), 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((70, 4), 5.0, device="cuda")
    need = fb4.fb4_cache8_attention_workspace(f.ctx, 4, 2, 128, 2, mq, mkv, 0)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    fb4.fb4_cache8_attention(f.ctx, big[:, 2:], 1280, 4, 70, f._cache(cache), table, table.shape[1], kv, qs, 2, mq, mkv, 128 ** -0.5,
                             True, 0, out[:, 128:], 768, 1, lse, ws if need else None, need)
    want = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(out[:63, 128:640].reshape(63, 4, 128), want[0]) and torch.equal(lse[:63], want[1])
    assert (out[63:] == 5).all() and (out[:, :128] == 5).all() and (out[:, 640:] == 5).all() and (lse[63:] == 5).all()


def test_the_plain_kernel_agrees(f):
    q, cache, table, kv, qs, mq, mkv = ref.setup([1, 40], [333, 80], 8, 2, 128, 16, seed=13)
    f.set_kernel_variant(1)
    got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, window=50)
    assert f.last_variant == "generic"
    f.set_kernel_variant(0)
    agree(got, ref.attend64(q, cache, table, kv, qs, 128 ** -0.5, True, 50, torch.bfloat16))


@pytest.mark.parametrize("block_size", [16, 32])
def test_a_server_step_by_step(block_size):
    """plan, append and attention: prompts, single tokens, drafted tokens of which some are rejected, an ended sequence whose place a new
    prompt takes; every step against float64 over what the cache holds, on a stream of its own.  Every context configuration will do"""
    f = fb4.Fb4(block_size=block_size)
    Hq, Hk, D, page, n, rows = 8, 2, 128, 16, 4, 80
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    gains = (1 + 0.1 * torch.randn(2, D, generator=g, device="cuda")).to(torch.bfloat16)
    tab = torch.from_numpy(attend_ref.rope_table(200, D, (64,))[0]).cuda()
    pages, cache = f.new_page_tables(n, 12, 30, page), f.new_cache8(30, page, Hk, D)
    steps = [([0, 0, 0, 0], [20, 3, 0, 41]), ([20, 3, 0, 41], [1, 1, 30, 1]), ([21, 4, 30, 42], [4, 4, 4, 4]), ([23, 8, 31, 42], [3, 1, 3, 2]), ([26, 0, 30, 44], [1, 37, 2, 1])]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        for keep, new in steps:
            plan = f.cache_plan(pages, ref.i32(new), rows, keep=ref.i32(keep))
            x = torch.randn(rows, Hq + 2 * Hk, D, generator=g, device="cuda").to(torch.bfloat16)
            q = f.cache8_append(cache, x[:, Hq:Hq + Hk], x[:, Hq + Hk:], pages.page_table, pages.kv_len, plan.q_start, 48, gains[1], 1e-6,
                                fb4.Rope(tab, plan.pos, [64]), q=x[:, :Hq], q_gain=gains[0])
            out = f.cache8_attention(q, cache, pages.page_table, pages.kv_len, plan.q_start, 48, 192)
            assert pages.kv_len.tolist() == [a + b for a, b in zip(keep, new)]
            agree(out, ref.attend64(q, cache, pages.page_table, pages.kv_len, plan.q_start, D ** -0.5, True, 0, torch.bfloat16))
            held = pages.page_table[[b for b in range(n) for _ in range(-(-int(pages.kv_len[b]) // page))], [i for b in range(n) for i in range(-(-int(pages.kv_len[b]) // page))]]
            assert held.unique().numel() == held.numel() == 30 - int(pages.n_free)       # no page belongs to two
            assert f.device_status == 0
    st.synchronize()
    f.close()


@pytest.mark.parametrize("q_len,kv_len,heads", [([1, 1], [1500, 200], (8, 2)), ([1, 1], [30000, 20000], (2, 1)), ([150, 40], [6000, 500], (2, 1))],
                         ids=["cluster", "few rows, workspace", "many rows, workspace"])
def test_captured_and_replayed(f, q_len, kv_len, heads):
    q, cache, table, kv, qs, mq, mkv = ref.setup(q_len, kv_len, *heads, 128, 16, seed=14)
    want = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=st):
        got = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    for _ in range(3):
        got[0].zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q2 = torch.randn_like(q)
    kv2 = kv // 2 + 75
    want = f.cache8_attention(q2, cache, table, kv2, qs, mq, mkv)
    q.copy_(q2)
    kv.copy_(kv2)
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0])


def test_two_calls_at_once_on_two_streams(f):
    args = [ref.setup([1, 2], [20000, 9000], 4, 1, 128, 16, seed=20), ref.setup([100, 60], [4000, 9000], 2, 2, 64, 32, seed=21)]
    want = [f.cache8_attention(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(8):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(f.cache8_attention(*args[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for a in got[i]:
            assert torch.equal(a[0], want[i][0]) and torch.equal(a[1], want[i][1])


@pytest.mark.parametrize("n_q", [1, 40])
def test_a_cache_whose_offsets_pass_32_bits(f, n_q):
    heads, page, D = 8, 64, 128
    n_pages = (1 << 32) // (heads * page * D) + 8000
    shape = (n_pages, heads, page, D)
    big = fb4.Cache8(*(torch.empty(s, dtype=torch.uint8, device="cuda") for s in (shape, (n_pages, heads, page // 16)) * 2))
    ids = [n_pages - 1, 0, n_pages - 7, 65536, 3]
    n = 5 * page - 9
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    kv = torch.randn(2, n, heads, D, generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn(n_q, heads, D, generator=g, device="cuda").to(torch.bfloat16)
    small = f.new_cache8(5, page, heads, D)
    one = ref.i32([n]), ref.i32([0, n]), n
    f.cache8_append(big, kv[0], kv[1], ref.i32([ids]), *one)
    f.cache8_append(small, kv[0], kv[1], ref.i32([[0, 1, 2, 3, 4]]), *one)
    a = f.cache8_attention(q, big, ref.i32([ids]), ref.i32([n]), ref.i32([0, n_q]), n_q, n)
    b = f.cache8_attention(q, small, ref.i32([[0, 1, 2, 3, 4]]), ref.i32([n]), ref.i32([0, n_q]), n_q, n)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(big.k[ids[0]], small.k[0]) and torch.equal(big.v_scale[ids[3]], small.v_scale[3])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_row_tiles_that_see_nothing(f, D, dtype):
    q, cache, table, kv, qs, mq, mkv = ref.setup([18, 33, 7] * 20, [2, 1, 60] * 20, 128, 8, D, 128, seed=30)
    want = ref.attend64(q[:58], cache, table[:3], kv[:3], qs[:4], D ** -0.5, True, 0, dtype)
    for _ in range(3):
        out, lse = f.cache8_attention(q, cache, table, kv, qs, mq, mkv, dtype=dtype)
        agree((out[:58], lse[:58]), want, dtype)
        o, l = out.view(20, 58, 128, D), lse.view(20, 58, 128)
        empty = torch.cat([torch.arange(16), 18 + torch.arange(32)]).cuda()
        assert not o[:, empty].any() and torch.isinf(l[:, empty]).all()


@pytest.mark.parametrize("name", SHAPES)
def test_outputs_and_workspace_stay_inside_their_arrays(f, name):
    from test_gpu_guard_bands import Guarded
    q, cache, table, kv, qs, mq, mkv = ref.setup(*SHAPES[name], seed=60)
    q_len, _, Hq, Hk, D, _ = SHAPES[name]
    T = q.shape[0]
    need = fb4.fb4_cache8_attention_workspace(f.ctx, Hq, Hk, D, len(q_len), mq, mkv, 0)
    out, lse, ws = Guarded(T * Hq * D * 2), Guarded(T * Hq * 4), Guarded(max(need, 256))
    fb4.fb4_cache8_attention(f.ctx, q, Hq * D, Hq, T, f._cache(cache), table, table.shape[1], kv, qs, len(q_len), mq, mkv, D ** -0.5, True, 0, out.view,
                             Hq * D, 1, lse.view, ws.view if need else None, need)
    torch.cuda.synchronize()
    for b, what in ((out, "out"), (lse, "lse"), (ws, "workspace")):
        b.check(what)
    want = f.cache8_attention(q, cache, table, kv, qs, mq, mkv)
    assert torch.equal(out.tensor(torch.bfloat16, (T, Hq, D)), want[0]) and torch.equal(lse.tensor(torch.float32, (T, Hq)), want[1])
