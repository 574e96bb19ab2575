"""Products with FB4 weights where every order of summation gives the same float32: whole numbers, whose sums stay below 2^24.  Nothing may be off, so a
run of channels that is left out, or taken twice, shows at any length: several chunks of x in shared memory, splits over a cluster, channels that end
inside a step, several tiles."""
import pytest
import torch

from paper_2603_02883_b200 import synth

BOOK = torch.from_numpy(synth.STANDIN_FORMATBOOK.astype("int64"))


def inputs(T, N, K, seed, device):
    """x in -2 .. 2, weights whose element scale is 1 (at most 15): a sum of magnitudes is at most 30 K"""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    x = torch.randint(-2, 3, (T, K), generator=g, device=device)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device=device, dtype=torch.uint8)
    dialect = torch.randint(0, 32, (N, K // 32), generator=g, device=device)
    bias = torch.randint(-100, 101, (N,), generator=g, device=device)
    return x, codes, dialect, bias


def values(codes, dialect):
    """float64 [N][K]"""
    book, did = BOOK.to(codes.device).double(), dialect.repeat_interleave(16, 1)
    out = torch.empty(codes.shape[0], codes.shape[1] * 2, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        nib = ((codes >> (4 * half)) & 15).long()
        out[:, half::2] = book[did, nib & 7] * (1 - 2 * (nib >> 3)).double()
    return out


def exact(x, codes, dialect):
    return x.double() @ values(codes, dialect).T


SIZES = [  # rows, N, K
    # mma.sync: one step, channels that end inside a step, x in one chunk and in several (1, 2, 5 and 8 rows: 256, 128, 32 steps of 128 channels at a time)
    (1, 1, 32), (1, 130, 4096), (1, 9, 300000), (2, 12, 131072 + 96), (3, 40, 100000), (5, 12, 65536), (8, 12, 65536 - 96), (7, 257, 1568), (8, 700, 12288),
    (12, 300, 4000), (16, 3000, 4096), (9, 1, 4064),
    # tcgen05: one chunk and many, steps of 256 channels that end early, one to several tiles and passes, one row of large weights
    (9, 12, 65536 - 96), (16, 40, 32768 + 160), (33, 70, 32768 - 96), (64, 40, 32768), (80, 33, 20000), (96, 300, 8224), (97, 130, 1024), (200, 300, 1056), (16, 4000, 8192),
    (61, 6152, 1568), (1, 32768, 4096), (4, 9000, 8256)]


@pytest.mark.gpu
@pytest.mark.parametrize("size", SIZES, ids=[".".join(map(str, s)) for s in SIZES])
def test_whole_numbers_are_exact(size):
    from paper_2603_02883_b200 import fb4
    T, N, K = size
    f = fb4.Fb4()
    x, codes, dialect, bias = inputs(T, N, K, T + N + K, "cuda")
    w, xb = fb4.Quantized(codes, (127 | (dialect << 8)).to(torch.int16)), x.to(torch.bfloat16)
    want = exact(x, codes, dialect)
    assert 30 * K < 1 << 24
    got = f.linear(xb, w, dtype=torch.float32)
    assert torch.equal(got.double(), want), f"{int((got.double() != want).sum())} of {want.numel()} differ"
    want = want + bias.double()
    assert torch.equal(f.linear(xb, w, bias.to(torch.bfloat16), dtype=torch.float32).double(), want)
    assert torch.equal(f.linear(xb, w, bias.to(torch.bfloat16)), want.to(torch.bfloat16))
    assert f.device_status == 0
    f.close()


@pytest.mark.parametrize("size", [s for s in SIZES if s[1] * s[2] < 2 << 20], ids=lambda s: ".".join(map(str, s)))
def test_a_missing_run_would_show(size):
    """planted in the oracle: with any run of 8 channels left out, or taken twice, some result differs"""
    T, N, K = size
    x, codes, dialect, _ = inputs(T, N, K, T + N + K, "cpu")
    v = values(codes, dialect)
    parts = torch.einsum("trc,nrc->rtn", x.double().view(T, K // 8, 8), v.view(N, K // 8, 8)) if T * N * K <= 1 << 26 else \
        torch.stack([(x[:2].double().view(-1, K // 8, 8) * v[n].view(K // 8, 8)).sum(-1).T for n in range(min(N, 12))], 2)
    missing = (parts == 0).flatten(1).all(1)
    # a run is missed where x is zero in every row, or its products cancel in every result: with one result only, by chance
    assert missing.double().mean() <= (0.2 if T * N == 1 else 0.0)
