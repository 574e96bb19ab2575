"""Out-of-bounds writes of the head norm and of the append: every output between two guard bands, ragged shapes, padded rows, slots
that are none."""
import numpy as np
import pytest
import torch

from paper_2603_02883_b200 import fb4
from test_gpu_guard_bands import Guarded
from test_gpu_norm_rope import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Hq,Hk,D,page,pairs,interleaved", [
    (1, 3, 1, 32, 16, (16,), False), (7, 1, 3, 96, 16, (16, 16, 16), True), (129, 5, 2, 128, 64, (64,), False), (50, 12, 12, 64, 32, (12, 10, 10), True),
    (3, 2, 5, 256, 128, (100, 28), False), (1025, 6, 1, 160, 16, (80,), True), (4000, 8, 2, 128, 16, (64,), True)])
def test_norm_and_append_stay_inside_their_buffers(T, Hq, Hk, D, page, pairs, interleaved):
    f = fb4.Fb4()
    x, g, rope, _, _ = make(T, Hq, Hk, D, pairs, interleaved, seed=T)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    n_pages = -(-T // page)
    q_out, k_out = Guarded(T * Hq * D * 2), Guarded(T * Hk * D * 2)
    want = f.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope)
    got = f.qk_norm_rope(q, k, g[0], g[1], 1e-6, rope, out=(q_out.tensor(torch.bfloat16, (T, Hq, D)), k_out.tensor(torch.bfloat16, (T, Hk, D))))
    torch.cuda.synchronize()
    q_out.check("q")
    k_out.check("k")
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    rows = n_pages * Hk * page
    held = [Guarded(rows * n) for n in (D // 2, D // 16, D // 2, D // 16)]
    shape = (n_pages, Hk, page)
    cache = fb4.Cache(held[0].tensor(torch.uint8, (*shape, D // 2)), held[1].tensor(torch.int16, (*shape, D // 32)),
                      held[2].tensor(torch.uint8, (*shape, D // 2)), held[3].tensor(torch.int16, (*shape, D // 32)))
    slot = np.random.default_rng(T).permutation(n_pages * page)[:T].astype(np.int64)
    if T > 5:
        slot[[1, T - 1]], slot[3], slot[4] = -1, n_pages * page, -2 ** 60
    q_out = Guarded(T * Hq * D * 2)
    fb4.fb4_cache_append(f.ctx, f._cache(cache), torch.from_numpy(slot).cuda(), k, x.stride(0), v, x.stride(0), T, g[1], 1e-6,
                         f._rope(rope, T, D), q, Hq, x.stride(0), g[0], q_out.view, Hq * D)
    torch.cuda.synchronize()
    for b, what in zip((*held, q_out), ("codes of k", "meta of k", "codes of v", "meta of v", "q of the append")):
        b.check(what)
    assert torch.equal(q_out.tensor(torch.bfloat16, (T, Hq, D)), want[0])
    assert f.device_status == (2 if T > 5 else 0)
    f.close()
