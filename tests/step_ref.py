"""Plain statements, on the CPU, of the operators of a decoding step: written from include/fb4.h, without the library's code."""
import numpy as np


def plan(page_table, kv_len, keep, new_len, free_pages, n_free, page, T):
    """sequence by sequence; -> (page_table, kv_len, free_pages, n_free, q_start, slot, pos, something was out of range)"""
    table, free = page_table.copy(), free_pages.copy()
    n, most = table.shape
    cap, bad = len(free), False
    up = lambda x: -(-x // page)  # noqa: E731
    count = min(max(int(n_free), 0), cap)
    bad |= count != int(n_free)
    lens, keeps, news = [], [], []
    for b in range(n):
        held = min(max(int(kv_len[b]), 0), most * page)
        bad |= held != int(kv_len[b])
        k = held if keep is None else int(keep[b])
        bad |= k < 0 or int(new_len[b]) < 0
        lens.append(held)
        keeps.append(min(max(k, 0), held))
        news.append(max(int(new_len[b]), 0))
    back = [table[b, i] for b in range(n) for i in range(up(keeps[b]), up(lens[b]))]
    top = count + len(back)
    for f, page_no in enumerate(back):
        if top - 1 - f < cap:
            free[top - 1 - f] = page_no
    bad |= top > cap
    top = min(top, cap)
    pages = rows = taken = 0
    q_start, kv = [0], []
    slot, pos = np.full(T, -1, np.int64), np.zeros(T, np.int32)
    for b in range(n):
        want = news[b] if keeps[b] + news[b] <= most * page else 0
        need = up(keeps[b] + want) - up(keeps[b])
        pages += need
        rows += want
        if pages > top or rows > T:
            want = 0
        for i in range(up(keeps[b]), up(keeps[b] + want)):
            table[b, i] = free[top - 1 - taken]
            taken += 1
        for i in range(want):
            p = keeps[b] + i
            slot[q_start[-1] + i] = int(table[b, p // page]) * page + p % page
            pos[q_start[-1] + i] = p
        kv.append(keeps[b] + want)
        q_start.append(q_start[-1] + want)
    return table, np.array(kv, np.int32), free, top - taken, np.array(q_start, np.int32), slot, pos, bool(bad)
