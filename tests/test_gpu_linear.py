"""Products with FB4 weights against float64: rows from one to many, sizes that no tile divides, strides, bias, output types, formatbooks,
splits, extreme scales, rows that are not finite; a quantized layer; refusals."""
import numpy as np
import pytest
import torch

import attend_ref as ref
from paper_2603_02883_b200 import fb4
from test_gpu_guard_bands import Guarded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def f():
    q = fb4.Fb4()
    yield q
    q.close()


def weights(N, K, seed=0, lo=112, hi=121):
    """any codes and dialects, scales between lo and hi"""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    sc = torch.randint(lo, hi, (N, K // 32), generator=g, device="cuda")
    return fb4.Quantized(codes, (sc | (torch.randint(0, 32, sc.shape, generator=g, device="cuda") << 8)).to(torch.int16))


def rows(T, K, pad=0, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    return torch.randn(T, K + pad, generator=g, device="cuda").to(torch.bfloat16)[:, :K]


def agree(got, x, w, bias, dtype):
    """one rounding to the output type, and float32 sums of K exact products: each addition off by half a step of what is summed
    so far (a whole one: the tensor cores may truncate), or by 2^-85"""
    v = ref.decode64(w.codes, w.meta)
    K = x.shape[1]
    want, size = x.double() @ v.T, x.double().abs() @ v.abs().T
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    step = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    tol = step * want.abs() + (K + 16) * (2.0 ** -23 * size * (1 + step) + 2.0 ** -85) + (2.0 ** -25 if dtype is torch.float16 else 0)
    assert got.dtype == dtype and got.shape == want.shape
    d = (got.double() - want).abs()
    assert (d <= tol).all(), f"off by {float((d / tol).max()):.3g} of what is allowed"


SIZES = [  # rows, N, K, padding of a row of x
    (1, 1, 32, 0), (1, 2048, 2048, 0), (1, 129, 96, 8), (2, 1000, 160, 0), (3, 16, 4096, 16), (7, 257, 1568, 0), (8, 128, 128, 0), (8, 5, 12288, 0), (9, 300, 64, 24),
    (15, 1, 480, 0), (16, 4096, 1024, 0), (17, 640, 544, 8), (31, 777, 992, 0), (32, 256, 16384, 0), (33, 1100, 32, 0), (61, 6152, 1568, 40), (64, 513, 2080, 0),
    (65, 130, 320, 0), (200, 300, 1056, 8), (1000, 33, 96, 0), (1, 20000, 64, 0), (5, 12, 65536, 0), (64, 40, 32768, 0), (12, 9000, 8192, 0)]


@pytest.mark.parametrize("size", SIZES, ids=[".".join(map(str, s)) for s in SIZES])
def test_matches_float64(f, size):
    T, N, K, pad = size
    x, w = rows(T, K, pad, seed=T), weights(N, K, seed=N)
    bias = torch.randn(N, device="cuda").to(torch.bfloat16) if (T + N) % 2 else None
    got = f.linear(x, w, bias)
    agree(got, x, w, bias, torch.bfloat16)
    assert torch.equal(got, f.linear(x, w, bias)) and f.device_status == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 10, 30, 64])
def test_output_types(f, T, dtype):
    x, w = rows(T, 1120, seed=T), weights(345, 1120, seed=T)
    bias = torch.randn(345, device="cuda").to(torch.bfloat16)
    agree(f.linear(x, w, bias, dtype=dtype), x, w, bias, dtype)


@pytest.mark.parametrize("T", [1, 6, 14, 40])
def test_scales_at_their_ends(f, T):
    for lo, hi, up in ((58, 62, 0), (186, 189, -60), (58, 189, -60)):
        x, w = rows(T, 256, seed=T), weights(70, 256, seed=T, lo=lo, hi=hi)
        x = (x.float() * 2.0 ** up).to(torch.bfloat16)
        agree(f.linear(x, w, dtype=torch.float32), x, w, None, torch.float32)
    x, w = rows(T, 256, seed=T), weights(70, 256, seed=T, lo=188, hi=189)
    x = (x.float() * 2.0 ** -60).to(torch.bfloat16)
    want = f.linear(x, w)
    w.meta.copy_((w.meta & ~255) | 240)                       # larger ones are read as 188
    assert torch.equal(f.linear(x, w), want)


@pytest.mark.parametrize("T", [3, 12, 50])
def test_a_row_that_is_not_finite_stays_alone(f, T):
    x, w = rows(T, 320, seed=T).clone(), weights(150, 320, seed=T)
    want = f.linear(x, w)
    x[0, 5], x[T - 1, 300] = float("nan"), float("inf")
    got = f.linear(x, w)
    assert torch.equal(got[1:T - 1], want[1:T - 1]) and torch.isnan(got[0]).all()
    zero = ref.decode64(w.codes, w.meta)[:, 300] == 0
    assert torch.isnan(got[T - 1][zero]).all() and torch.isinf(got[T - 1][~zero].float()).all()
    x.zero_()
    assert not f.linear(x, w).any()


def test_another_formatbook(f):
    book = np.sort(np.stack([np.random.default_rng(i).choice(np.arange(1, 16), 7, replace=False) for i in range(32)]), 1)
    book = np.concatenate([np.zeros((32, 1), np.int64), book], 1).astype(np.uint8)
    g = fb4.Fb4(formatbook=book)
    x, w = rows(20, 640), weights(200, 640)
    kept = ref.BOOK
    try:
        ref.BOOK = book
        agree(g.linear(x, w), x, w, None, torch.bfloat16)
    finally:
        ref.BOOK = kept
    g.close()


@pytest.mark.parametrize("T", [1, 20])
def test_a_quantized_layer(f, T):
    """weights through the offline quantizer, the activation through the online one and its decode: what the MXFP8 operands of the same
    tensors give, here without an operand being written out"""
    w = f.quantize_weights((torch.randn(384, 1024, device="cuda") / 32).to(torch.bfloat16))
    x = f.dequantize(f.quantize(rows(T, 1024)), torch.bfloat16)
    agree(f.linear(x, w), x, w, None, torch.bfloat16)
    dense = f.dequantize(w)
    assert (f.linear(x, w, dtype=torch.float32) - x.float() @ dense.t()).abs().max() <= 2 * 1040 * 2.0 ** -23 * float((x.float().abs() @ dense.abs().t()).max())


def test_offsets_beyond_32_bits(f):
    """9 GB of codes: the last rows agree with the same weights on their own"""
    N, K = 1100000, 16384
    codes = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda").random_(0, 256)
    meta = torch.randint(0x0070, 0x0079, (N, K // 32), device="cuda", dtype=torch.int16)
    x = rows(2, K)
    big = f.linear(x, fb4.Quantized(codes, meta), dtype=torch.float32)
    part = slice(N - 300, N)
    w = fb4.Quantized(codes[part].clone(), meta[part].clone())
    agree(big[:, part], x, w, None, torch.float32)


@pytest.mark.parametrize("T", [1, 9, 33])
def test_captured_on_another_stream_and_strided_output(f, T):
    x, w = rows(T, 2080, 8, seed=T).clone(), weights(500, 2080, seed=T)
    want = f.linear(x, w)
    out = Guarded(T * 600 * 2)
    o = out.tensor(torch.bfloat16, (T, 600))
    o.zero_()
    st, gr = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(gr, stream=st):
        fb4.fb4_linear(f.ctx, x, T, 2080, x.stride(0), w.codes, w.meta, 500, None, o, 600, 1)
    for _ in range(2):
        gr.replay()
    torch.cuda.synchronize()
    out.check("out")
    assert torch.equal(o[:, :500], want) and not o[:, 500:].any()
    x.mul_(2)
    gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(o[:, :500], f.linear(x, w))


@pytest.mark.parametrize("size", [(1, 12288, 12288), (5, 9000, 8192), (12, 9000, 8192), (16, 3000, 4096), (14, 1500, 8192), (32, 12288, 8192), (64, 7000, 8192), (96, 9500, 2048)], ids=lambda s: ".".join(map(str, s)))
def test_many_items_again_and_again(f, size):
    """several tiles, chunks and laps of every ring, with other traffic in memory between: each run gives the same bits"""
    T, N, K = size
    x, w = rows(T, K, seed=T), weights(N, K, seed=N)
    first = f.linear(x, w, dtype=torch.float32)
    agree(first, x, w, None, torch.float32)
    other = torch.ones(48 << 20, device="cuda")
    for i in range(60):
        if i % 3 == 0:
            other.mul_(1.0001)
        assert torch.equal(f.linear(x, w, dtype=torch.float32), first), f"run {i}"
    assert f.device_status == 0


def test_two_calls_at_once(f):
    args = [(rows(1, 4096, seed=1), weights(3000, 4096, seed=1)), (rows(40, 4096, seed=2), weights(1000, 4096, seed=2))]
    want = [f.linear(*a) for a in args]
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for _ in range(6):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(f.linear(*args[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[i]) for i in range(2) for a in got[i])


def test_empty_calls_and_refusals(f):
    x, w = rows(4, 64), weights(10, 64)
    assert f.linear(x[:0], w).shape == (0, 10) and f.linear(x, fb4.Quantized(w.codes[:0], w.meta[:0])).shape == (4, 0)
    z = fb4.Fb4(block_size=16)
    with pytest.raises(fb4.Fb4Error) as e:
        z.linear(x, w)
    assert e.value.code == fb4.ERR_INVALID_ARG
    z.close()
    with pytest.raises(fb4.Fb4Error) as e:
        f.linear(torch.zeros(4, 68, dtype=torch.bfloat16, device="cuda")[:, 1:65], w)
    assert e.value.code == fb4.ERR_ALIGN
