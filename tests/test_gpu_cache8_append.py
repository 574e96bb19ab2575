"""fb4_cache8_append bit for bit against its statement: lengths, places inside a block, held tokens, head dimensions, pairings, strides,
padded rows, positions below zero, bad pages, extreme values; the decode; outputs that stay inside their arrays; refusals."""
import numpy as np
import pytest
import torch

import attend_ref
import cache8_ref as ref
from paper_2603_02883_b200 import fb4, synth
from test_gpu_guard_bands import Guarded
from test_gpu_norm_rope import as_f32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def f():
    q = fb4.Fb4()
    yield q
    q.close()


def host(cache):
    return [t.cpu().numpy().copy() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)]


def appended(f, cache, x, g, rope, plain, Hq, Hk, table, kv, qs, max_q, eps=1e-6):
    """makes the call and checks all of it; -> q"""
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    want = host(cache)
    t, n, s = table.cpu().numpy(), kv.cpu().numpy(), qs.cpu().numpy()
    out = f.cache8_append(cache, k, v, table, kv, qs, max_q, g[1], eps, rope, q=q if Hq else None, q_gain=g[0])
    ref.append(attend_ref.norm_rotate_f32(as_f32(k.contiguous()), as_f32(g[1]), eps, plain), want[0], want[1], t, n, s)
    ref.append(as_f32(v.contiguous()), want[2], want[3], t, n, s)
    for name, a, b in zip(("k", "k_scale", "v", "v_scale"), host(cache), want):
        assert np.array_equal(a, b), name
    if Hq:
        rows = np.zeros(len(x), bool)                        # rows at positions from 0 on
        for b in range(len(n)):
            rows[s[b] + max(0, s[b + 1] - s[b] - n[b]):s[b + 1]] = True
        want_q = attend_ref.norm_rotate_f32(as_f32(q.contiguous()), as_f32(g[0]), eps, plain)
        got = out.cpu().view(torch.int16).numpy().view(np.uint16)
        assert np.array_equal(got[rows], synth.f32_to_bf16_bits(want_q)[rows])
    return out


CASES = [
    # new tokens, cached tokens with them, q heads, k heads, D, page, pairs of the axes, interleaved
    ([1], [1], 32, 8, 128, 16, (64,), False), ([1], [16], 1, 1, 32, 16, (16,), True), ([1] * 5, [17, 1, 15, 1000, 32], 4, 2, 128, 32, (64,), False),
    ([3, 0, 20], [10, 50, 20], 4, 4, 64, 16, (32,), True), ([17], [31], 2, 1, 128, 16, (22, 21, 21), True), ([18], [33], 2, 2, 128, 64, (22, 21, 21), False),
    ([100, 37], [133, 37], 0, 3, 96, 32, (16, 16, 16), False), ([200], [1200], 3, 3, 256, 128, (128,), True), ([33, 65], [77, 65], 5, 1, 160, 16, (7, 30, 43), False),
    ([2, 2, 2], [2, 18, 17], 1, 1, 224, 16, (50, 62), True), ([700, 5], [5000, 5], 2, 2, 64, 4096, (8, 8, 9, 7), False), ([16, 32, 48], [16, 48, 64], 12, 12, 128, 64, (64,), True),
    ([1] * 70, list(range(1, 71)), 8, 8, 128, 16, (64,), False), ([300, 1, 1, 1], [300, 7, 8, 9], 2, 1, 32, 16, (16,), False),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_bit_for_bit(f, case):
    q_len, kv_len, Hq, Hk, D, page, pairs, inter = case
    T = sum(q_len) + 3                                        # rows of no sequence
    x, g, rope, plain, _ = make(T, Hq, Hk, D, pairs, inter, seed=T + D)
    table, n_pages, kv, qs = ref.tables(q_len, kv_len, page, seed=T)
    cache = ref.random_cache(n_pages, Hk, page, D, seed=T)
    appended(f, cache, x, g, rope, plain, Hq, Hk, table, kv, qs, max(q_len))
    before = host(cache)
    appended(f, cache, x, g, rope, plain, Hq, Hk, table, kv, qs, max(q_len) + 40)        # again: nothing moves
    assert all(np.array_equal(a, b) for a, b in zip(before, host(cache)))
    assert f.device_status == 0


@pytest.mark.parametrize("n_seqs", [3, 33, 1100])
def test_one_long_prompt_among_short_ones(f, n_seqs):
    """CTAs are dealt out by rows, the sequence being looked up"""
    q_len = [i % 4 for i in range(n_seqs)]
    q_len[n_seqs // 2] = 1500
    kv_len = [a + 5 * i % 23 for i, a in enumerate(q_len)]
    T = sum(q_len)
    x, g, rope, plain, _ = make(T, 1, 1, 64, (32,), False, seed=n_seqs)
    table, n_pages, kv, qs = ref.tables(q_len, kv_len, 16, seed=n_seqs)
    appended(f, ref.random_cache(n_pages, 1, 16, 64, seed=1), x, g, rope, plain, 1, 1, table, kv, qs, 1500)
    assert f.device_status == 0


def test_without_norm_and_rotation_q_in_place_and_padded_strides(f):
    x, g, _, _, _ = make(40, 2, 2, 128, (64,), False, seed=9)
    table, n_pages, kv, qs = ref.tables([25, 15], [30, 200], 32, seed=9)
    cache = ref.random_cache(n_pages, 2, 32, 128, seed=9)
    want = host(cache)
    wide = torch.zeros(40, 9, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 1:7] = x
    f.cache8_append(cache, wide[:, 3:5], wide[:, 5:7], table, kv, qs, 25)
    for i, part in ((0, x[:, 2:4]), (2, x[:, 4:6])):
        ref.append(as_f32(part.contiguous()), want[i], want[i + 1], *(t.cpu().numpy() for t in (table, kv, qs)))
    assert all(np.array_equal(a, b) for a, b in zip(host(cache), want))
    q = wide[:, 1:3].clone().contiguous()
    expect = f.cache8_append(cache, wide[:, 3:5], wide[:, 5:7], table, kv, qs, 25, q=q, q_gain=g[0])
    fb4.fb4_cache8_append(f.ctx, f._cache(cache), table, table.shape[1], kv, qs, 2, 25, wide[:, 3:], 9 * 128, wide[:, 5:], 9 * 128, 40, None, 1e-6, None,
                          q, 2, 256, g[0], q, 256)
    assert torch.equal(q, expect)


def test_extreme_values(f):
    """zeros, subnormals, the limits of the exponent, a value at 127.5 steps, infinities that stay in their block"""
    D, Hk = 64, 1
    v = torch.zeros(16 * 9, 1, D, device="cuda")
    v[16:32] = 2.0 ** -130
    v[32:48] = 2.0 ** -70
    v[48:64] = 3.0e38
    v[64:80] = 127.5
    v[80:96] = torch.linspace(-127.49, 127.49, 16 * D, device="cuda").view(16, 1, D)
    v[96:112] = (torch.arange(16 * D, device="cuda").view(16, 1, D) % 255 - 127).float() + 0.5        # ties
    v[112:128] = 2.0 ** 65 * 0.99
    v[128:] = torch.randn(16, 1, D, device="cuda")
    v = v.to(torch.bfloat16)
    k = torch.randn(16 * 9, 1, D, device="cuda").to(torch.bfloat16)
    table, n_pages, kv, qs = ref.tables([16 * 9], [16 * 9], 16, seed=2)
    cache = ref.random_cache(n_pages, Hk, 16, D, seed=2)
    want = host(cache)
    f.cache8_append(cache, k, v, table, kv, qs, 16 * 9)
    for i, part in ((0, k), (2, v)):
        ref.append(as_f32(part), want[i], want[i + 1], *(t.cpu().numpy() for t in (table, kv, qs)))
    assert all(np.array_equal(a, b) for a, b in zip(host(cache), want))
    k[5, 0, 3], v[40, 0, 0], k[100, 0, 9] = float("inf"), float("nan"), float("-inf")
    f.cache8_append(cache, k, v, table, kv, qs, 16 * 9)
    clean = [b for b in range(9) if b not in (0, 2, 6)]
    pages = table[0].cpu().numpy()
    for a, b in zip(host(cache), want):
        assert np.array_equal(a[pages[clean]], b[pages[clean]])
    assert f.device_status == 0


def test_token_by_token_is_off_by_one_step_at_most(f):
    """a block that grows sixteen times; at once it is off by half a step"""
    T, D = 64, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    k = torch.randn(T, 2, D, generator=g, device="cuda") * torch.linspace(0.1, 9, T, device="cuda")[:, None, None]
    k = k.to(torch.bfloat16)
    table, n_pages, _, _ = ref.tables([T], [T], 32, seed=3)
    for steps, most in (([T], 0.5), ([1] * T, 1.0), ([5, 1, 30, 28], 1.0)):
        cache, at = f.new_cache8(n_pages, 32, 2, D), 0
        for n in steps:
            f.cache8_append(cache, k[at:at + n], k[at:at + n], table, ref.i32([at + n]), ref.i32([0, n]), n)
            at += n
        got = f.cache8_values(cache)[0][table[0].long()].transpose(1, 2).flatten(0, 1)                  # [T][H][D]
        step = torch.exp2(cache.k_scale[table[0].long()].float() - 127).transpose(1, 2).flatten(0, 1).repeat_interleave(16, 0)[..., None]
        assert ((got - k.float()).abs() <= most * step).all()


def test_positions_below_zero_and_bad_pages():
    f = fb4.Fb4()
    x, g, rope, plain, _ = make(60, 2, 2, 64, (32,), False, seed=11)
    table, n_pages, kv, qs = ref.tables([30, 30], [20, 90], 16, seed=11)
    cache = ref.random_cache(n_pages, 2, 16, 64, seed=11)
    appended(f, cache, x, g, rope, plain, 2, 2, table, kv, qs, 30)
    assert f.device_status == 0
    table[1, 4] = n_pages                                     # its tokens go nowhere, and are reported
    appended(f, cache, x, g, rope, plain, 2, 2, table, kv, qs, 30)
    assert f.device_status == 2
    f.close()


def test_lengths_outside_their_bounds_and_bad_positions_are_reported():
    for what in ("kv_len", "q_start", "pos"):
        f = fb4.Fb4()
        x, g, rope, plain, _ = make(8, 1, 1, 64, (32,), False, seed=12)
        table, n_pages, kv, qs = ref.tables([5, 3], [64, 20], 16, seed=12)
        cache = ref.random_cache(n_pages, 1, 16, 64, seed=12)
        if what == "kv_len":
            kv[0] = 65
        elif what == "q_start":
            qs[2] = 400
        else:
            rope.pos[2] = -1
        f.cache8_append(cache, x[:, 1:2], x[:, 2:3], table, kv, qs, 5, g[1], 1e-6, rope, q=x[:, :1], q_gain=g[0])
        assert f.device_status == 2
        f.close()


@pytest.mark.parametrize("D,page", [(32, 16), (128, 64), (96, 16), (256, 32)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_decode(f, D, page, dtype):
    cache = ref.random_cache(7, 3, page, D, seed=D, lo=0 if dtype is not torch.float16 else 100, hi=256 if dtype is not torch.float16 else 135)
    for got, codes, scale in zip(f.cache8_values(cache, dtype), (cache.k, cache.v), (cache.k_scale, cache.v_scale)):
        assert got.dtype == dtype and torch.equal(got.double(), ref.decode64(codes, scale).to(dtype).double())
    k, v = f.cache8_values(f.new_cache8(2, 16, 1, 32))
    assert not k.any() and not v.any()


@pytest.mark.parametrize("T,Hq,Hk,D,page,pairs", [(1, 3, 1, 32, 16, (16,)), (37, 2, 3, 128, 16, (64,)), (50, 1, 2, 96, 64, (48,)), (20, 2, 1, 256, 32, (128,))])
def test_outputs_stay_inside_their_arrays(f, T, Hq, Hk, D, page, pairs):
    x, g, rope, plain, _ = make(T, Hq, Hk, D, pairs, False, seed=T)
    n_pages = -(-T // page)
    held = [Guarded(n_pages * Hk * page * D), Guarded(n_pages * Hk * page // 16), Guarded(n_pages * Hk * page * D), Guarded(n_pages * Hk * page // 16)]
    shape = (n_pages, Hk, page)
    cache = fb4.Cache8(held[0].tensor(torch.uint8, (*shape, D)), held[1].tensor(torch.uint8, (n_pages, Hk, page // 16)),
                       held[2].tensor(torch.uint8, (*shape, D)), held[3].tensor(torch.uint8, (n_pages, Hk, page // 16)))
    table = ref.i32([list(range(n_pages - 1, -1, -1))])
    q_out = Guarded(T * Hq * D * 2)
    fb4.fb4_cache8_append(f.ctx, f._cache(cache), table, n_pages, ref.i32([T]), ref.i32([0, T]), 1, T, x[:, Hq:], x.stride(0), x[:, Hq + Hk:], x.stride(0),
                          T, g[1], 1e-6, f._rope(rope, T, D), x, Hq, x.stride(0), g[0], q_out.view, Hq * D)
    values = [Guarded(n_pages * Hk * page * D * 2) for _ in range(2)]
    fb4.fb4_cache8_values(f.ctx, f._cache(cache), values[0].view, values[1].view, 1)
    torch.cuda.synchronize()
    for b in (*held, q_out, *values):
        b.check("append")
    assert f.device_status == 0


def test_captured_on_another_stream_and_replayed(f):
    x, g, rope, plain, _ = make(9, 4, 2, 128, (64,), False, seed=15)
    table, n_pages, kv, qs = ref.tables([4, 5], [40, 60], 16, seed=15)
    cache = ref.random_cache(n_pages, 2, 16, 128, seed=15)
    twin = fb4.Cache8(*(t.clone() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)))
    args = (x[:, 4:6], x[:, 6:8], table, kv, qs, 9, g[1], 1e-6, rope)
    want = f.cache8_append(twin, *args, q=x[:, :4], q_gain=g[0])
    st, gr = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(gr, stream=st):
        got = f.cache8_append(cache, *args, q=x[:, :4], q_gain=g[0])
    for _ in range(2):
        gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(np.array_equal(a, b) for a, b in zip(host(cache), host(twin)))
    kv -= 7
    want = f.cache8_append(twin, *args, q=x[:, :4], q_gain=g[0])
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(np.array_equal(a, b) for a, b in zip(host(cache), host(twin)))
