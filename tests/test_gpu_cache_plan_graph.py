"""fb4_cache_plan in a CUDA graph in the forms that larger steps take: a cluster (more than 512 sequences or 2048 rows), and the rows in a second
kernel that is launched early (more than 8192 rows); replayed on other lengths, with what follows in the graph reading the plan."""
import numpy as np
import pytest
import torch

import step_ref
from paper_2603_02883_b200 import fb4
from test_gpu_cache_plan import dev, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,most,T", [(700, 3, 2000), (40, 90, 3000), (2000, 2, 8192), (2000, 14, 20000), (3, 30000, 60000), (8192, 3, 16500)])
def test_captured_and_replayed_on_other_lengths(n, most, T):
    f = fb4.Fb4()
    r = np.random.RandomState(n)
    max_pages = 4 + -(-6 * most // 16)
    table, kv, free, spare = state(r, n, 16, 40, max_pages, n * max_pages)
    pt = fb4.PageTables(dev(table), dev(kv), dev(free), dev(np.array([spare], np.int32)), 16)
    new, keep = dev(np.zeros(n, np.int32)), dev(kv)
    st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=st):
        plan = f.cache_plan(pt, new, T, keep=keep)
        copies = [t.clone() for t in (plan.q_start, plan.slot, plan.pos, pt.kv_len, pt.page_table)]      # read right behind it
        again = f.cache_plan(pt, new, T, keep=keep)                                                    # the same step again: the same plan
    now = (table, kv, free, spare)
    for step in range(4):
        add = r.randint(0, most + 1, n).astype(np.int32)
        stay = np.maximum(now[1] - r.randint(0, 5, n), 0).astype(np.int32)
        if step == 2:
            stay[::3] = 0
        new.copy_(dev(add))
        keep.copy_(dev(stay))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = step_ref.plan(now[0], now[1], stay, add, now[2], now[3], 16, T)
        for name, got, i in (("q_start", copies[0], 4), ("slot", copies[1], 5), ("pos", copies[2], 6), ("kv_len", copies[3], 1), ("page_table", copies[4], 0),
                             ("q_start again", again.q_start, 4), ("slot again", again.slot, 5), ("pos again", again.pos, 6), ("kv_len again", pt.kv_len, 1),
                             ("page_table again", pt.page_table, 0)):
            assert np.array_equal(got.cpu().numpy(), want[i]), f"step {step}: {name}"
        assert int(pt.n_free[0]) == want[3] and np.array_equal(pt.free_pages.cpu().numpy()[:want[3]], want[2][:want[3]])
        now = want[:4]
    assert f.device_status == 0
    del g
    f.close()
