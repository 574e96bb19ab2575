"""fb4_cache8_append with q_start outside its bounds: clamped and reported alike, whether the CTAs are dealt out by sequence or by rows."""
import numpy as np
import pytest
import torch

import cache8_ref as ref
from paper_2603_02883_b200 import fb4

pytestmark = pytest.mark.gpu

# (q_start as given, q_start as it is clamped) of 40 sequences over 64 rows
GOOD = [min(64, 2 * b) for b in range(41)]
BAD = {
    "first far below zero": ([-1000] + GOOD[1:], GOOD),
    "first one below zero": ([-1] + GOOD[1:], GOOD),
    "from the middle on far above": (GOOD[:25] + [10 ** 6] * 16, GOOD[:25] + [64] * 16),
    "all far above": ([10 ** 6] * 41, [64] * 41),
    "one that falls": (GOOD[:10] + [10 ** 9] + GOOD[11:], None),
    "the last above": (GOOD[:40] + [65], GOOD),
}


@pytest.mark.parametrize("max_q", [17, 4096])
@pytest.mark.parametrize("name", BAD)
def test_q_start_outside_its_bounds_is_clamped_and_reported(name, max_q):
    """max_q 17: CTAs by sequence, 4096: by rows, the sequence being looked up"""
    given, clamped = BAD[name]
    f = fb4.Fb4()
    n_q = np.diff(GOOD if clamped is None else clamped)
    kv_len = np.maximum(n_q, 0) + 21
    table, n_pages, kv, _ = ref.tables(n_q, kv_len, 16, seed=1)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    k, v = (torch.randn(64, 2, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    cache = ref.random_cache(n_pages, 2, 16, 64, seed=2)
    want = fb4.Cache8(*(t.clone() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)))
    if clamped is not None:
        f.cache8_append(want, k, v, table, kv, ref.i32(clamped), max_q)
        assert f.device_status == 0
    f.cache8_append(cache, k, v, table, kv, ref.i32(given), max_q)
    assert f.device_status == 2
    if clamped is not None:
        for part in ("k", "k_scale", "v", "v_scale"):
            assert torch.equal(getattr(cache, part), getattr(want, part)), part
    f.close()
