"""Append to the paged FB4 cache: the written blocks bit for bit against the oracle's quantization of the float32 result of
the stated norm and rotation; untouched slots, padded rows, bad slots, page sizes, head layouts, refusals."""
import numpy as np
import pytest
import torch

import attend_ref as ref
from oracle import fb4_oracle as orc
from paper_2603_02883_b200 import fb4, synth
from test_gpu_norm_rope import as_f32, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


def blocks(y):
    """oracle codes and meta of float32 [T][H][D]"""
    T, H, D = y.shape
    z = orc.quantize_f32(np.ascontiguousarray(y.reshape(T * H, D)), ref.BOOK)
    return z.codes.reshape(T, H, D // 2), z.meta.reshape(T, H, D // 32)


def check(cache, before, slot, T, want, what):
    codes, meta = (getattr(cache, what + "_codes").cpu().numpy(), getattr(cache, what + "_meta").cpu().numpy().view(np.uint16))
    c0, m0 = (getattr(before, what + "_codes").cpu().numpy().copy(), getattr(before, what + "_meta").cpu().numpy().view(np.uint16).copy())
    page = codes.shape[2]
    for t in range(T):
        s = int(slot[t])
        if 0 <= s < codes.shape[0] * page:
            c0[s // page, :, s % page], m0[s // page, :, s % page] = want[0][t], want[1][t]
    assert np.array_equal(codes, c0) and np.array_equal(meta, m0)


def clone(c):
    return fb4.Cache(*(getattr(c, f).clone() for f in ("k_codes", "k_meta", "v_codes", "v_meta")))


@pytest.mark.parametrize("T,Hq,Hk,D,page,pairs,interleaved", [
    (1, 32, 8, 128, 16, (64,), False), (1, 0, 1, 32, 16, (16,), True), (45, 12, 12, 128, 64, (22, 21, 21), True),
    (333, 8, 2, 64, 32, (32,), False), (17, 5, 5, 96, 128, (16, 16, 16), False), (6, 4, 2, 256, 16, (128,), True),
    (29, 3, 3, 160, 4096, (40, 40), False), (3000, 16, 4, 128, 256, (64,), False), (64, 7, 1, 64, 16, (32,), True)])
def test_blocks_match_the_oracle(q32, T, Hq, Hk, D, page, pairs, interleaved):
    x, g, rope, plain, _ = make(T, Hq, Hk, D, pairs, interleaved, seed=11 + T)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    n_pages = -(-T // page) + 2
    rng = np.random.default_rng(T)
    slot = rng.permutation(n_pages * page)[:T].astype(np.int64)
    if T > 10:
        slot[[2, T - 1]] = -1                                    # rows that pad the batch
    cache = ref.random_cache(q32, n_pages, Hk, page, D, seed=5)
    before = clone(cache)
    qo = q32.cache_append(cache, torch.from_numpy(slot).cuda(), k, v, g[1], 1e-6, rope, q=q if Hq else None, q_gain=g[0] if Hq else None)
    check(cache, before, slot, T, blocks(ref.norm_rotate_f32(as_f32(k.contiguous()), as_f32(g[1]), 1e-6, plain)), "k")
    check(cache, before, slot, T, blocks(as_f32(v.contiguous())), "v")
    if Hq:
        assert torch.equal(qo, q32.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope)[0])
    else:
        assert qo is None
    assert q32.device_status == 0


def test_values_are_what_the_quantizer_gives(q32):
    """without norm and rotation an append is fb4_quantize of the rows, and cache_values is fb4_dequantize of the cache"""
    x, *_ = make(200, 0, 4, 128, (64,), False, seed=2)
    k, v = x[:, :4], x[:, 4:]
    cache = q32.new_cache(13, 16, 4, 128)
    assert not q32.cache_values(cache)[0].any()
    slot = torch.arange(200, device="cuda")
    assert q32.cache_append(cache, slot, k, v) is None
    kv = q32.cache_values(cache, torch.bfloat16)
    for held, src in zip(kv, (k, v)):
        rows = src.reshape(800, 128).contiguous()
        want = q32.dequantize(q32.quantize(rows), torch.bfloat16).view(200, 4, 128)
        got = held.transpose(1, 2).reshape(-1, 4, 128)
        assert torch.equal(got[:200], want) and not got[200:].any()


def test_bad_slots_and_positions_are_left_out_and_reported():
    q = fb4.Fb4()
    x, g, rope, plain, _ = make(70, 0, 2, 64, (32,), False, seed=9)
    slot = np.arange(70, dtype=np.int64)
    slot[[0, 13, 69]] = [-2, 5 * 16, 2 ** 62]
    cache = ref.random_cache(q, 5, 2, 16, 64, seed=1)
    before = clone(cache)
    rope.pos[20] = 97
    plain = (plain[0], rope.pos.cpu().numpy(), plain[2], plain[3])
    q.cache_append(cache, torch.from_numpy(slot).cuda(), x[:, :2], x[:, 2:], g[1], 1e-6, rope)
    check(cache, before, slot, 70, blocks(ref.norm_rotate_f32(as_f32(x[:, :2].contiguous()), as_f32(g[1]), 1e-6, plain)), "k")
    check(cache, before, slot, 70, blocks(as_f32(x[:, 2:].contiguous())), "v")
    assert q.device_status == 2
    q.close()


def test_an_infinity_stays_in_its_own_row(q32):
    x, g, rope, plain, _ = make(40, 2, 2, 128, (64,), False, seed=10)
    clean = q32.new_cache(3, 16, 2, 128)
    slot = torch.arange(40, device="cuda")
    qa = q32.cache_append(clean, slot, x[:, 2:4], x[:, 4:], g[1], 1e-6, rope, q=x[:, :2], q_gain=g[0])
    x[7, 2, 5], x[9, 4, 100], x[11, 0, 0] = float("inf"), float("nan"), float("-inf")
    dirty = q32.new_cache(3, 16, 2, 128)
    qb = q32.cache_append(dirty, slot, x[:, 2:4], x[:, 4:], g[1], 1e-6, rope, q=x[:, :2], q_gain=g[0])
    for f, row, head in (("k_codes", 7, 0), ("k_meta", 7, 0), ("v_codes", 9, 0), ("v_meta", 9, 0)):
        a, b = getattr(clean, f).transpose(1, 2).reshape(48, 2, -1), getattr(dirty, f).transpose(1, 2).reshape(48, 2, -1)
        same = (a == b).all(-1)
        same[row, head] = True
        assert same.all()
    keep = torch.ones(40, 2, dtype=torch.bool, device="cuda")
    keep[11, 0] = False
    assert torch.equal(qa[keep], qb[keep])


def test_refusals(q32):
    x, g, rope, plain, _ = make(8, 2, 2, 64, (32,), False, seed=8)
    cache = q32.new_cache(4, 16, 2, 64)
    c = q32._cache(cache)
    r = q32._rope(rope, 8, 64)
    slot = torch.arange(8, device="cuda")
    o = torch.empty(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    ok = dict(cache=c, slot=slot, k=x[:, 2:4], k_ld=384, v=x[:, 4:], v_ld=384, T=8, k_gain=g[1], eps=1e-6, rope=r, q=x, q_heads=2,
              q_ld=384, q_gain=g[0], q_out=o, q_out_ld=128)

    def code(ctx=q32.ctx, **change):
        try:
            fb4.fb4_cache_append(ctx, **{**ok, **change})
        except fb4.Fb4Error as e:
            return e.code
        return 0

    def other(**change):
        d = fb4.Fb4Cache(*(getattr(c, f) for f, _ in c._fields_))
        for f, v in change.items():
            setattr(d, f, v)
        return d
    assert code() == 0 and code(T=0) == 0
    assert code(T=-1) == fb4.ERR_SHAPE and code(slot=None) == fb4.ERR_INVALID_ARG and code(cache=None) == fb4.ERR_INVALID_ARG
    assert code(slot=slot.data_ptr() + 4) == fb4.ERR_ALIGN and code(k=x.data_ptr() + 2) == fb4.ERR_ALIGN and code(v_ld=100) == fb4.ERR_SHAPE
    assert code(k=None) == fb4.ERR_INVALID_ARG and code(v=None) == fb4.ERR_INVALID_ARG and code(q_out=None) == fb4.ERR_INVALID_ARG
    assert code(eps=float("inf")) == fb4.ERR_INVALID_ARG and code(q_heads=-1) == fb4.ERR_INVALID_ARG
    for change in (dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=8192), dict(n_pages=0), dict(n_heads=0), dict(head_dim=40),
                   dict(head_dim=288), dict(n_pages=2 ** 40)):
        assert code(cache=other(**change)) == fb4.ERR_SHAPE, change
    assert code(cache=other(k_meta=None)) == fb4.ERR_INVALID_ARG and code(cache=other(v_codes=c.v_codes + 8)) == fb4.ERR_ALIGN
    for cfg in (dict(block_size=16), dict(num_groups=32), dict(select_mode=1), dict(exp_min=-15, exp_max=16)):
        z = fb4.Fb4(**cfg)
        assert code(ctx=z.ctx) == fb4.ERR_INVALID_ARG
        z.close()
    with pytest.raises(ValueError):
        q32.cache_append(cache, slot.int(), x[:, 2:4], x[:, 4:])
    with pytest.raises(ValueError):
        q32.cache_append(cache, slot, x[:, 2:5], x[:, 4:])
    with pytest.raises(ValueError):
        q32.cache_append(fb4.Cache(cache.k_codes, cache.k_meta[:, :1], cache.v_codes, cache.v_meta), slot, x[:, 2:4], x[:, 4:])


def test_without_q_heads_its_pointers_are_ignored(q32):
    x, g, rope, plain, _ = make(20, 0, 2, 64, (32,), False, seed=13)
    a, b = q32.new_cache(2, 16, 2, 64), q32.new_cache(2, 16, 2, 64)
    slot, odd = torch.arange(20, device="cuda"), g.data_ptr() + 2
    q32.cache_append(a, slot, x[:, :2], x[:, 2:], g[1], 1e-6, rope)
    fb4.fb4_cache_append(q32.ctx, q32._cache(b), slot, x, 256, x[:, 2:], 256, 20, g[1], 1e-6, q32._rope(rope, 20, 64), odd, 0, -1, odd, odd, -1)
    for f in ("k_codes", "k_meta", "v_codes", "v_meta"):
        assert torch.equal(getattr(a, f), getattr(b, f))


def test_another_formatbook(q32):
    """a formatbook that the packed tables hold is used; one with more than 8 candidates to a stage-1 group is refused"""
    base = np.array([[0, 1, 2, 3, 5, 7, 9, 8 + d % 8] for d in range(32)], np.uint8)
    base[:, 6] = np.minimum(base[:, 6], base[:, 7] - 1)
    base[:, 5] = np.minimum(base[:, 5], base[:, 6] - 1)
    mask = np.array([0xff << (8 * (k % 4)) for k in range(32)], np.uint32)
    assert (np.diff(base.astype(int), axis=1) > 0).all()
    f = fb4.Fb4(formatbook=base, stage1_mask=mask)
    x, *_ = make(50, 0, 2, 128, (64,), False, seed=14)
    cache = f.new_cache(4, 16, 2, 128)
    f.cache_append(cache, torch.arange(50, device="cuda"), x[:, :2], x[:, 2:])
    rows = as_f32(x[:, 2:].contiguous()).reshape(100, 128)
    z = orc.quantize_f32(np.ascontiguousarray(rows), base, stage1=mask)
    got = cache.v_codes.transpose(1, 2).reshape(64, 2, 64)[:50].reshape(100, 64).cpu().numpy()
    assert np.array_equal(got, z.codes)
    q = torch.randn(3, 4, 128, device="cuda").to(torch.bfloat16)
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([50], dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    out, _ = f.cache_attention(q, cache, table, *lens, 3, 50, dtype=torch.float32)
    kv = [t.double().transpose(1, 2).reshape(64, 2, 128)[:50].repeat_interleave(2, 1) for t in f.cache_values(cache)]
    p = torch.einsum("ihd,jhd->hij", q.double(), kv[0]) * 128 ** -0.5
    p = p.masked_fill(torch.arange(50, device="cuda") > 47 + torch.arange(3, device="cuda")[:, None], float("-inf")).softmax(-1)
    want, size = torch.einsum("hij,jhd->ihd", p, kv[1]), torch.einsum("hij,jhd->ihd", p, kv[1].abs())
    # probabilities rounded to bfloat16, 2^-8 of each term; float32 sums of 128 and of 50 terms move them by less than 2^-10 more
    # what underflows: the second product is summed times 2^-64 in float32, whose smallest step is 2^-149, so each of its 50
    # additions can lose 2^-85 of the result; a probability below 2^-126 is 0, and 50 of those times a value below 2^41 are less
    # than 50 * 2^-85 again
    assert kv[1].abs().max() < 2.0 ** 41
    assert ((out.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -10) * size + 2 * 50 * 2.0 ** -85).all()
    f.close()
    wide = fb4.Fb4(stage1_mask=np.full(32, 0x1ff, np.uint32))
    with pytest.raises(fb4.Fb4Error) as e:
        wide.cache_append(wide.new_cache(4, 16, 2, 128), torch.arange(50, device="cuda"), x[:, :2], x[:, 2:])
    assert e.value.code == fb4.ERR_INVALID_ARG
    wide.close()
