"""fb4_cache_plan against the statement of tests/step_ref.py: every entry equal, whatever the lengths."""
import numpy as np
import pytest
import torch

import step_ref
from paper_2603_02883_b200 import fb4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    f = fb4.Fb4()
    yield f
    f.close()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def state(r, n, page, held_max, max_pages, spare):
    """a consistent server: tables, lengths, free list"""
    kv = r.randint(0, held_max + 1, n).astype(np.int32)
    pages = -(-kv.astype(np.int64) // page)
    total = int(pages.sum())
    perm = r.permutation(total + spare).astype(np.int32)
    table = np.full((n, max_pages), -7, np.int32)
    at = 0
    for b in range(n):
        table[b, :pages[b]] = perm[at:at + pages[b]]
        at += pages[b]
    free = np.full(total + spare, -9, np.int32)
    free[:spare] = perm[at:]
    return table, kv, free, spare


def check(q, table, kv, free, n_free, page, keep, new, T, again=False):
    pt = fb4.PageTables(dev(table), dev(kv), dev(free), dev(np.array([n_free], np.int32)), page)
    for _ in range(2 if again else 1):
        plan = q.cache_plan(pt, dev(new), T, keep=None if keep is None else dev(keep))
    want = step_ref.plan(table, kv, keep, new, free, n_free, page, T)
    for name, x, y in zip(("page_table", "kv_len", "free_pages", "n_free", "q_start", "slot", "pos"),
                          (pt.page_table, pt.kv_len, pt.free_pages, pt.n_free, plan.q_start, plan.slot, plan.pos), want):
        x = x.cpu().numpy()
        if name == "n_free":
            assert int(x[0]) == y
        elif name == "free_pages":                          # what lies above the top is left over
            assert np.array_equal(x[:want[3]], y[:want[3]]), name
        else:
            assert x.dtype == y.dtype and np.array_equal(x, y), name
    return want, pt, plan


@pytest.mark.parametrize("n,page,held,new_max,slack", [
    (0, 16, 0, 0, 5), (1, 16, 0, 1, 0), (1, 16, 5000, 1, 3), (2, 32, 31, 2, 0), (31, 16, 100, 5, 7), (128, 16, 40, 1, 0), (129, 64, 300, 9, 1),
    (512, 16, 33, 3, 11), (513, 16, 33, 3, 0), (1024, 16, 20, 4, 3), (1025, 16, 20, 4, 3), (3000, 128, 500, 20, 60), (7, 4096, 9000, 9000, 100), (5, 16, 3, 3000, 0)])
def test_keep_and_add(q, n, page, held, new_max, slack):
    r = np.random.RandomState(n * 7 + page)
    max_pages = max(1, -(-(held + new_max) // page))
    table, kv, free, spare = state(r, n, page, held, max_pages, 3 + n * (-(-new_max // page) + 1))
    keep = np.maximum(kv - r.randint(0, 40, n), 0).astype(np.int32)
    keep[::5] = 0
    new = r.randint(0, new_max + 1, n).astype(np.int32)
    T = int(new.sum()) + slack
    want, _, _ = check(q, table, kv, free, spare, page, keep, new, T)
    assert want[4][-1] == new.sum()                         # everybody is served here
    check(q, table, kv, free, spare, page, keep, new, T, again=True)
    check(q, table, kv, free, spare, page, None, np.minimum(new, max_pages * page - kv).astype(np.int32), T)
    assert q.device_status == 0


@pytest.mark.parametrize("n", [1, 40, 700, 2100])
@pytest.mark.parametrize("short", ["pages", "rows", "both", "nothing left"])
def test_not_enough_for_all(q, n, short):
    r = np.random.RandomState(n)
    table, kv, free, spare = state(r, n, 16, 90, 12, 4 * n)
    keep = np.maximum(kv - r.randint(0, 20, n), 0).astype(np.int32)
    new = r.randint(0, 70, n).astype(np.int32)
    if short in ("pages", "both"):
        spare //= 3
    if short == "nothing left":
        spare, keep = 0, kv.copy()
    T = int(new.sum()) // 2 if short in ("rows", "both") else int(new.sum()) + 5
    check(q, table, kv, free, spare, 16, keep, new, T, again=True)
    assert q.device_status == 0


def test_a_table_that_has_no_room(q):
    """such a sequence gets nothing and stands in nobody's way"""
    r = np.random.RandomState(3)
    table, kv, free, spare = state(r, 50, 16, 60, 4, 400)
    new = np.where(np.arange(50) % 3 == 0, 1 << 30, 2).astype(np.int32)
    kv[:] = np.minimum(kv, 62)
    want, _, _ = check(q, table, kv, free, spare, 16, None, new, 200)
    assert want[4][-1] == 2 * int((np.arange(50) % 3 != 0).sum())
    new[:] = 2147483647
    want, _, _ = check(q, table, kv, free, spare, 16, None, new, 200)
    assert want[4][-1] == 0


def test_no_rows_and_no_list(q):
    table, kv, free, spare = state(np.random.RandomState(4), 5, 16, 60, 4, 4)
    check(q, table, kv, free, spare, 16, None, np.ones(5, np.int32), 0)
    pt = fb4.PageTables(dev(table), dev(kv), torch.empty(0, dtype=torch.int32, device="cuda"), dev(np.zeros(1, np.int32)), 16)
    plan = q.cache_plan(pt, dev(np.zeros(5, np.int32)), 3)
    assert plan.slot.tolist() == [-1] * 3 and plan.q_start.tolist() == [0] * 6 and pt.kv_len.tolist() == kv.tolist()


def test_the_largest_number_of_sequences_and_many_rows(q):
    r = np.random.RandomState(5)
    n = 8192
    table, kv, free, spare = state(r, n, 16, 20, 4, n)
    new = r.randint(0, 9, n).astype(np.int32)
    keep = np.maximum(kv - 3, 0).astype(np.int32)
    check(q, table, kv, free, spare, 16, keep, new, int(new.sum()) + 1000)
    table, kv, free, spare = state(r, 3, 16, 20, 40000, 90000)              # three long prompts
    check(q, table, kv, free, spare, 16, None, np.array([600001, 0, 333333], np.int32), 933334 + 31)
    assert q.device_status == 0


def test_values_out_of_range_are_clamped_and_reported():
    r = np.random.RandomState(6)
    cases = []
    for what in ("kv_len", "negative kv_len", "keep", "new_len", "n_free", "negative n_free", "full list"):
        table, kv, free, spare = state(r, 20, 16, 60, 6, 50)
        keep, new, page_list = kv.copy(), np.full(20, 3, np.int32), free
        if what == "kv_len":
            kv[3] = 6 * 16 + 1
        elif what == "negative kv_len":
            kv[3] = -1
        elif what == "keep":
            keep[5] = -2
        elif what == "new_len":
            new[5] = -2
        elif what == "n_free":
            spare = len(free) + 1
        elif what == "negative n_free":
            spare = -1
        else:
            keep[:] = 0
            free = free[:40]
            spare = 35
        cases.append((table, kv, free, spare, keep, new))
    for table, kv, free, spare, keep, new in cases:
        f = fb4.Fb4()
        want, _, _ = check(f, table, kv, free, spare, 16, keep, new, 100)
        assert want[-1] and f.device_status == 2
        f.close()


def test_captured_and_replayed_on_other_lengths(q):
    r = np.random.RandomState(7)
    table, kv, free, spare = state(r, 33, 16, 60, 12, 300)
    pt = fb4.PageTables(dev(table), dev(kv), dev(free), dev(np.array([spare], np.int32)), 16)
    new, keep = dev(np.zeros(33, np.int32)), dev(kv)
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q.cache_plan(pt, new, 100, keep=keep)
    side.synchronize()
    with torch.cuda.graph(g, stream=side):
        plan = q.cache_plan(pt, new, 100, keep=keep)
    now = (table, kv, free, spare)
    for step in range(4):
        add = r.randint(0, 4, 33).astype(np.int32)
        stay = np.maximum(now[1] - r.randint(0, 3, 33), 0).astype(np.int32)
        new.copy_(dev(add))
        keep.copy_(dev(stay))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = step_ref.plan(now[0], now[1], stay, add, now[2], now[3], 16, 100)
        assert np.array_equal(plan.slot.cpu().numpy(), want[5]) and np.array_equal(plan.pos.cpu().numpy(), want[6])
        assert np.array_equal(pt.kv_len.cpu().numpy(), want[1]) and np.array_equal(pt.page_table.cpu().numpy(), want[0])
        now = want[:4]
    assert q.device_status == 0


def test_outputs_stay_inside_their_arrays(q):
    r = np.random.RandomState(8)
    for n, T in ((3, 17), (700, 1500)):
        table, kv, free, spare = state(r, n, 16, 60, 6, 2 * n)
        guard = 64
        room = lambda count, dtype: torch.full((count + 2 * guard,), 77, dtype=dtype, device="cuda")  # noqa: E731
        q_start, slot, pos = room(n + 1, torch.int32), room(T, torch.int64), room(T, torch.int32)
        mid = lambda t: t[guard:-guard]  # noqa: E731
        d = [dev(table), dev(kv), dev(free), dev(np.array([spare], np.int32))]
        new = dev(np.full(n, 2, np.int32))
        fb4.fb4_cache_plan(q.ctx, d[0], 6, 16, d[1], None, new, n, d[2], len(free), d[3], T, mid(q_start), mid(slot), mid(pos))
        want = step_ref.plan(table, kv, None, np.full(n, 2, np.int32), free, spare, 16, T)
        for t, w in ((q_start, want[4]), (slot, want[5]), (pos, want[6])):
            t = t.cpu().numpy()
            assert (t[:guard] == 77).all() and (t[-guard:] == 77).all() and np.array_equal(t[guard:-guard], w)
    assert q.device_status == 0
