"""A decoding step of one attention layer: plan, projection by FB4 weights, append and attention over the 8-bit cache, projection back; recorded
into a CUDA graph that plans itself from the lengths it finds, step after step, beside the same calls made one by one."""
import pytest
import torch

import attend_ref
from paper_2603_02883_b200 import fb4

pytestmark = pytest.mark.gpu

Hq, Hk, D, PAGE, C = 8, 2, 128, 16, 512


def layer(f, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    w_in, w_out = f.quantize_weights(new((Hq + 2 * Hk) * D, C) * 0.1), f.quantize_weights(new(C, Hq * D) * 0.1)
    return w_in, w_out, new(C), 1 + new(D) * 0.1, 1 + new(D) * 0.1


def step(f, weights, pages, cache, tab, x, new_len, keep, max_q):
    w_in, w_out, bias, q_gain, k_gain = weights
    rows = x.shape[0]
    plan = f.cache_plan(pages, new_len, rows, keep=keep)
    h = f.linear(x, w_in).view(rows, Hq + 2 * Hk, D)
    q = f.cache8_append(cache, h[:, Hq:Hq + Hk], h[:, Hq + Hk:], pages.page_table, pages.kv_len, plan.q_start, max_q, k_gain, 1e-6,
                        fb4.Rope(tab, plan.pos, [64]), q=h[:, :Hq], q_gain=q_gain)
    out, _ = f.cache8_attention(q, cache, pages.page_table, pages.kv_len, plan.q_start, max_q, 256)
    return f.linear(out.view(rows, Hq * D), w_out, bias)


@pytest.mark.parametrize("n,drafts", [(1, 1), (5, 1), (4, 3), (40, 2)])
def test_a_recorded_step_equals_the_calls_one_by_one(n, drafts):
    f = fb4.Fb4()
    weights = layer(f, n)
    tab = torch.from_numpy(attend_ref.rope_table(256, D, (64,))[0]).cuda()
    rows = n * drafts
    g = torch.Generator(device="cuda")
    g.manual_seed(n + 7)
    prompts = [int(v) for v in torch.randint(1, 60, (n,), generator=g, device="cuda")]
    x0 = torch.randn(sum(prompts), C, generator=g, device="cuda").to(torch.bfloat16)
    new0, new = torch.tensor(prompts, dtype=torch.int32, device="cuda"), torch.full((n,), drafts, dtype=torch.int32, device="cuda")
    sides = []
    for _ in range(2):
        pages, cache = f.new_page_tables(n, 16, 16 * n, PAGE), f.new_cache8(16 * n, PAGE, Hk, D)
        first = step(f, weights, pages, cache, tab, x0, new0, None, 64)
        sides.append((pages, cache, first))
    assert torch.equal(sides[0][2], sides[1][2])
    x, keep = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=st):
        got = step(f, weights, sides[0][0], sides[0][1], tab, x, new, keep, drafts)
    for i in range(6):
        x.copy_(torch.randn(rows, C, generator=g, device="cuda"))
        # all that is held, less some of the drafts of the step before
        rejected = torch.randint(0, drafts, (n,), generator=g, device="cuda") if i else torch.zeros(n, device="cuda")
        keep.copy_(sides[1][0].kv_len - rejected)
        graph.replay()
        want = step(f, weights, sides[1][0], sides[1][1], tab, x, new, keep, drafts)
        torch.cuda.synchronize()
        assert torch.isfinite(want).all() and torch.equal(got, want), f"step {i}"
        assert torch.equal(sides[0][0].kv_len, keep + new)
        for a, b in ((sides[0][0].page_table, sides[1][0].page_table), (sides[0][0].n_free, sides[1][0].n_free), (sides[0][1].k, sides[1][1].k),
                     (sides[0][1].v, sides[1][1].v), (sides[0][1].k_scale, sides[1][1].k_scale)):
            assert torch.equal(a, b)
    assert f.device_status == 0
    del graph
    f.close()
