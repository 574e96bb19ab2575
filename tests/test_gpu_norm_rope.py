"""Per-head norm with the position rotation: bit for bit against the stated float32 order, and against the formulas in
float64; head dimensions, pairings, axes, strides, in place, positions outside the table, refusals."""
import numpy as np
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q32():
    q = fb4.Fb4()
    yield q
    q.close()


def bits(x):
    return torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)


def as_f32(t):
    return ref.bf16_to_f32(t.cpu().view(torch.int16).numpy().view(np.uint16))


def make(T, Hq, Hk, D, axis_pairs, interleaved, n_pos=97, seed=0):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((T, Hq + 2 * Hk, D)) * np.exp(rng.standard_normal((T, 1, 1)) * 2)).astype(np.float32)
    x[rng.random(x.shape) < 0.01] *= 50
    gains = (1 + 0.3 * rng.standard_normal((2, D))).astype(np.float32)
    pos = rng.integers(0, n_pos, (T, len(axis_pairs))).astype(np.int32)
    table, freq = ref.rope_table(n_pos, D, axis_pairs)
    xd = bits(synth.f32_to_bf16_bits(x))
    gd = bits(synth.f32_to_bf16_bits(gains))
    rope = fb4.Rope(torch.from_numpy(table).cuda(), torch.from_numpy(pos).cuda(), list(axis_pairs), interleaved)
    return xd, gd, rope, (table, pos, list(axis_pairs), interleaved), freq


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,pairs", [
    (1, 32, 8, 128, (64,)), (1, 1, 1, 32, (16,)), (37, 12, 12, 128, (22, 21, 21)), (5, 7, 1, 64, (32,)), (9, 3, 2, 96, (16, 16, 16)),
    (4, 2, 3, 256, (128,)), (3, 5, 1, 160, (7, 30, 43)), (700, 5, 5, 64, (8, 8, 9, 7)), (2, 1, 1, 224, (50, 62)), (1300, 40, 8, 128, (64,))])
def test_matches_the_stated_order_bit_for_bit(q32, T, Hq, Hk, D, pairs, interleaved):
    x, g, rope, plain, freq = make(T, Hq, Hk, D, pairs, interleaved, seed=T + D)
    q, k = x[:, :Hq], x[:, Hq:Hq + Hk]
    qo, ko = q32.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope)
    for got, src, gain in ((qo, q, g[0]), (ko, k, g[1])):
        want = ref.norm_rotate_f32(as_f32(src.contiguous()), as_f32(gain), 1e-6, plain)
        assert np.array_equal(got.cpu().view(torch.int16).numpy().view(np.uint16), synth.f32_to_bf16_bits(want))
        # half a step of the result, and the float32 steps before it: the norm 2^-20, the rotation 2^-22 of the pair, the table 2^-24
        exact = ref.norm_rotate_f64(as_f32(src.contiguous()), as_f32(gain), 1e-6, freq, plain[1], plain[2], interleaved)
        top = np.abs(exact).max(-1, keepdims=True)
        assert (np.abs(as_f32(got) - exact) <= 2.0 ** -8 * np.abs(exact) + 2.0 ** -18 * top).all()
    assert q32.device_status == 0


def test_without_norm_without_rotation_and_one_side_only(q32):
    x, g, rope, plain, _ = make(33, 4, 2, 128, (64,), False, seed=3)
    q, k = x[:, :4], x[:, 4:6]
    qo, ko = q32.qk_norm_rope(q, k, None, g[1], 1e-5, rope)
    assert np.array_equal(as_f32(qo), ref.bf16_to_f32(synth.f32_to_bf16_bits(ref.norm_rotate_f32(as_f32(q.contiguous()), None, 0, plain))))
    qo, ko = q32.qk_norm_rope(q, k, g[0], None, 1e-5, None)
    assert torch.equal(ko, k)
    assert np.array_equal(as_f32(qo), ref.bf16_to_f32(synth.f32_to_bf16_bits(ref.norm_rotate_f32(as_f32(q.contiguous()), as_f32(g[0]), 1e-5, None))))
    qo, ko = q32.qk_norm_rope(q, k[:, :0], g[0], None, 1e-5, rope)
    assert ko.shape == (33, 0, 128) and qo.abs().sum() > 0
    empty = q32.qk_norm_rope(q[:0], k[:0], g[0], g[1], 1e-5, fb4.Rope(rope.table, rope.pos[:0], [64]))
    assert empty[0].shape == (0, 4, 128)


def test_zero_rows_and_huge_rows(q32):
    x, g, rope, plain, _ = make(6, 2, 1, 64, (32,), True, seed=4)
    x[0] = 0
    x[1] *= 2.0 ** 60
    x[2] *= 2.0 ** -70
    q, k = x[:, :2], x[:, 2:3]
    qo, _ = q32.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope)
    with np.errstate(over="ignore"):
        want = ref.norm_rotate_f32(as_f32(q.contiguous()), as_f32(g[0]), 1e-6, plain)
    assert np.array_equal(qo.cpu().view(torch.int16).numpy().view(np.uint16), synth.f32_to_bf16_bits(want))
    assert not qo[0].any()


def test_in_place_on_a_packed_projection_leaves_v_alone(q32):
    x, g, rope, plain, _ = make(130, 6, 2, 128, (22, 21, 21), True, seed=5)
    before = x.clone()
    q, k = x[:, :6], x[:, 6:8]
    want = q32.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope)
    q32.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope, out=(q, k))
    assert torch.equal(x[:, :6], want[0]) and torch.equal(x[:, 6:8], want[1]) and torch.equal(x[:, 8:], before[:, 8:])


def test_position_outside_the_table_counts_as_zero_and_is_reported():
    q32 = fb4.Fb4()
    x, g, rope, plain, _ = make(40, 2, 1, 64, (10, 22), False, seed=6)
    rope.pos[3, 1], rope.pos[7, 0], rope.pos[39, 1] = -1, 97, 2 ** 31 - 1
    plain = (plain[0], rope.pos.cpu().numpy(), plain[2], plain[3])
    qo, _ = q32.qk_norm_rope(x[:, :2], x[:, 2:3], g[0], g[1], 1e-6, rope)
    want = ref.norm_rotate_f32(as_f32(x[:, :2].contiguous()), as_f32(g[0]), 1e-6, plain)
    assert np.array_equal(qo.cpu().view(torch.int16).numpy().view(np.uint16), synth.f32_to_bf16_bits(want))
    assert q32.device_status == 2
    q32.close()


def test_guard_rows_around_a_strided_output(q32):
    x, g, rope, plain, _ = make(50, 3, 1, 64, (32,), False, seed=7)
    big = torch.full((50, 5 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, ko = big[:, 64:256].view(50, 3, 64), torch.empty(50, 1, 64, dtype=torch.bfloat16, device="cuda")
    want = q32.qk_norm_rope(x[:, :3], x[:, 3:4], g[0], g[1], 1e-6, rope)
    q32.qk_norm_rope(x[:, :3], x[:, 3:4], g[0], g[1], 1e-6, rope, out=(qo, ko))
    assert torch.equal(qo, want[0]) and (big[:, :64] == 7).all() and (big[:, 256:] == 7).all()


def test_refusals(q32):
    x, g, rope, plain, _ = make(8, 2, 1, 64, (32,), False, seed=8)
    q, k = x[:, :2], x[:, 2:3]
    r = q32._rope(rope, 8, 64)
    o = torch.empty(8, 3, 64, dtype=torch.bfloat16, device="cuda")
    ok = dict(q=q, q_heads=2, q_ld=256, k=k, k_heads=1, k_ld=256, T=8, D=64, q_gain=g[0], k_gain=g[1], eps=1e-6, rope=r,
              q_out=o, q_out_ld=128, k_out=o, k_out_ld=128)

    def code(**change):
        try:
            fb4.fb4_qk_norm_rope(q32.ctx, **{**ok, **change})
        except fb4.Fb4Error as e:
            return e.code
        return 0
    p = lambda t, off: t.data_ptr() + off  # noqa: E731
    assert code(D=48) == fb4.ERR_SHAPE and code(D=288) == fb4.ERR_SHAPE and code(T=-1) == fb4.ERR_SHAPE
    assert code(q_ld=120) == fb4.ERR_SHAPE and code(q_out_ld=64) == fb4.ERR_SHAPE and code(q_ld=260) == fb4.ERR_ALIGN
    assert code(q=p(x, 2)) == fb4.ERR_ALIGN and code(k_out=p(o, 8)) == fb4.ERR_ALIGN and code(q_gain=p(g, 2)) == fb4.ERR_ALIGN
    assert code(eps=-1.0) == fb4.ERR_INVALID_ARG and code(eps=float("nan")) == fb4.ERR_INVALID_ARG
    assert code(q=None) == fb4.ERR_INVALID_ARG and code(k_out=None) == fb4.ERR_INVALID_ARG and code(q_heads=-1) == fb4.ERR_INVALID_ARG
    assert code(q_out=q, q_out_ld=128) == fb4.ERR_INVALID_ARG              # in place with another stride
    for change in (dict(n_axes=0), dict(n_axes=5), dict(interleaved=2), dict(table=None), dict(pos=None), dict(pairs=(-1, 33))):
        bad = fb4.Fb4Rope(r.table, r.n_pos, r.pos, change.get("n_axes", 2), (fb4.ctypes.c_int32 * 4)(*change.get("pairs", (16, 16))),
                          change.get("interleaved", 0))
        for f in ("table", "pos"):
            if f in change:
                setattr(bad, f, None)
        assert code(rope=bad) == fb4.ERR_INVALID_ARG
    assert code(rope=fb4.Fb4Rope(r.table, r.n_pos, r.pos, 1, (fb4.ctypes.c_int32 * 4)(31), 0)) == fb4.ERR_SHAPE
    assert code(rope=fb4.Fb4Rope(r.table, 0, r.pos, 1, (fb4.ctypes.c_int32 * 4)(32), 0)) == fb4.ERR_SHAPE
    assert code(rope=fb4.Fb4Rope(r.table + 8, r.n_pos, r.pos, 1, (fb4.ctypes.c_int32 * 4)(32), 0)) == fb4.ERR_ALIGN
    with pytest.raises(ValueError):
        q32.qk_norm_rope(q.float(), k)
    with pytest.raises(ValueError):
        q32.qk_norm_rope(x.transpose(0, 1), k)
    with pytest.raises(ValueError):
        q32.qk_norm_rope(q, k[:4])
    with pytest.raises(ValueError):
        q32.qk_norm_rope(q, k, rope=fb4.Rope(rope.table, rope.pos[:5], [32]))
    with pytest.raises(ValueError):
        q32.qk_norm_rope(q.cpu(), k)


def test_pointers_of_a_side_without_heads_are_ignored(q32):
    """not read and not checked: here a gain that is not even aligned"""
    x, g, rope, plain, _ = make(20, 2, 2, 64, (32,), False, seed=12)
    q, k = x[:, :2], x[:, 2:4]
    want = q32.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope)
    r, odd = q32._rope(rope, 20, 64), g.data_ptr() + 2
    for side in (0, 1):
        out = torch.zeros(20, 2, 64, dtype=torch.bfloat16, device="cuda")
        real = lambda src, gain: [(src, 2, 384), gain, (out, 128)]  # noqa: E731
        none = [(odd, 0, -1), odd, (odd, -1)]
        a, b = (real(q, g[0]), none) if side == 0 else (none, real(k, g[1]))
        fb4.fb4_qk_norm_rope(q32.ctx, *a[0], *b[0], 20, 64, a[1], b[1], 1e-6, r, *a[2], *b[2])
        assert torch.equal(out, want[side])
