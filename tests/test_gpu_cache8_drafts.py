"""Drafted tokens of large values that are rejected: what they leave in a block of the 8-bit cache."""
import numpy as np
import pytest
import torch

import cache8_ref as ref
from paper_2603_02883_b200 import fb4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first,drafts,after", [(5, 1, 1), (5, 3, 40), (12, 4, 2), (16, 1, 3), (3, 13, 20)])
def test_rejected_drafts_of_large_values(first, drafts, after):
    """A block's exponent does not fall while tokens stand in front of the new ones, so rejected drafts count: what is kept is off by one step of the block's
    exponent at most, what comes behind by half a step; from a block's first place on it is that of the new tokens alone."""
    f = fb4.Fb4()
    g = torch.Generator(device="cuda")
    g.manual_seed(first)
    new = lambda n, s: (torch.randn(n, 2, 64, generator=g, device="cuda") * s).to(torch.bfloat16)      # noqa: E731
    pages, cache = f.new_page_tables(1, 8, 8, 16), f.new_cache8(8, 16, 2, 64)
    held, keep = [], 0
    for x, stay in ((new(first, 1.0), 0), (new(drafts, 1000.0), first), (new(after, 1.0), first)):
        plan = f.cache_plan(pages, ref.i32([len(x)]), len(x), keep=ref.i32([stay]))
        f.cache8_append(cache, x, x, pages.page_table, pages.kv_len, plan.q_start, len(x))
        held = held[:stay] + list(x)
    x = torch.stack(held).float()
    total = first + after
    assert int(pages.kv_len[0]) == total
    ids = pages.page_table[0, :-(-total // 16)].long()
    for got, scale in zip(f.cache8_values(cache), (cache.k_scale, cache.v_scale)):
        got = got[ids].transpose(1, 2).flatten(0, 1)[:total]
        step = torch.exp2(scale[ids].float() - 127).transpose(1, 2).flatten(0, 1).repeat_interleave(16, 0)[:total, :, None]
        off = (got - x).abs()
        assert (off[:first] <= step[:first]).all() and (off[first:] <= 0.5 * step[first:]).all()
        top = (x.abs().amax(2), step[..., 0])
        for block in range(-(-total // 16)):
            rows = slice(16 * block, min(16 * block + 16, total))
            tight = torch.from_numpy(np.array([2.0 ** ref.exponent(float(t)) for t in top[0][rows].amax(0)])).cuda()
            grown = (step[rows][0, :, 0] > tight).any()
            assert bool(grown) == (16 * block < first < 16 * block + 16), f"block {block}"
    assert f.device_status == 0
    f.close()
