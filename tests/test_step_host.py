"""Refusals of the calls of a decoding step, without a device: the C entry points on a context made by hand (nothing may reach a launch),
and the binding on tensors of the CPU, its calls recorded instead of made."""
import pytest
import torch

from paper_2603_02883_b200 import fb4
from test_attention_binding import context
from test_attention_host import run

PLAN = r"""
  int32_t* w = reinterpret_cast<int32_t*>(room);
  int64_t* slot = reinterpret_cast<int64_t*>(room);
  ctx.plan_error = cudaErrorInvalidConfiguration;
  auto plan = [&](int32_t* table, int max_pages, int page, int32_t* kv, int32_t* add, int n, int32_t* free_pages, int cap, int32_t* n_free, int64_t T,
                  int32_t* start, int64_t* slots, int32_t* pos) {
    return fb4_cache_plan(&ctx, table, max_pages, page, kv, 0, add, n, free_pages, cap, n_free, T, start, slots, pos, 0);
  };
  if (plan(w, 4, 16, w, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_CUDA || fb4_last_cuda_error() != (int)cudaErrorInvalidConfiguration) return 1;
  if (fb4_cache_plan(0, w, 4, 16, w, 0, w, 2, w, 8, w, 10, w, slot, w, 0) != FB4_ERR_INVALID_ARG) return 2;
  for (int page : {0, 8, 15, 24, 8192, -16})
    if (plan(w, 4, page, w, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_SHAPE) return 3;
  if (plan(w, -1, 16, w, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_SHAPE || plan(w, (1 << 26) + 1, 16, w, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_SHAPE) return 4;
  if (plan(w, 1 << 26, 16, w, w, 31, w, 8, w, 10, w, slot, w) != FB4_ERR_CUDA || plan(w, 1 << 26, 16, w, w, 32, w, 8, w, 10, w, slot, w) != FB4_ERR_SHAPE) return 5;
  if (plan(w, 4, 16, w, w, -1, w, 8, w, 10, w, slot, w) != FB4_ERR_SHAPE || plan(w, 4, 16, w, w, FB4_PLAN_MAX_SEQS + 1, w, 8, w, 10, w, slot, w) != FB4_ERR_SHAPE) return 6;
  if (plan(w, 4, 16, w, w, 2, w, -1, w, 10, w, slot, w) != FB4_ERR_SHAPE) return 7;
  if (plan(w, 4, 16, w, w, 2, w, 8, w, -1, w, slot, w) != FB4_ERR_SHAPE || plan(w, 4, 16, w, w, 2, w, 8, w, 1LL << 31, w, slot, w) != FB4_ERR_SHAPE) return 8;
  if (plan(0, 4, 16, w, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_INVALID_ARG || plan(w, 4, 16, 0, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_INVALID_ARG) return 9;
  if (plan(w, 4, 16, w, 0, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_INVALID_ARG || plan(w, 4, 16, w, w, 2, 0, 8, w, 10, w, slot, w) != FB4_ERR_INVALID_ARG) return 10;
  if (plan(w, 4, 16, w, w, 2, w, 8, 0, 10, w, slot, w) != FB4_ERR_INVALID_ARG || plan(w, 4, 16, w, w, 2, w, 8, w, 10, 0, slot, w) != FB4_ERR_INVALID_ARG) return 11;
  if (plan(0, 0, 16, w, w, 2, 0, 0, w, 10, w, 0, 0) != FB4_ERR_CUDA || plan(0, 4, 16, 0, 0, 0, 0, 0, w, 0, w, 0, 0) != FB4_ERR_CUDA) return 12;   // nothing to point to
  int32_t* odd = reinterpret_cast<int32_t*>(room + 2);
  int64_t* half = reinterpret_cast<int64_t*>(room + 4);
  if (plan(odd, 4, 16, w, w, 2, w, 8, w, 10, w, slot, w) != FB4_ERR_ALIGN || plan(w, 4, 16, w, w, 2, w, 8, w, 10, w, half, w) != FB4_ERR_ALIGN) return 13;
  if (ctx.launches != 0) return 14;
  puts("ok");
  return 0;
}
"""


def test_plan_refusals(tmp_path):
    run(tmp_path, PLAN)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def tables(monkeypatch, n=3, max_pages=4):
    monkeypatch.setattr(fb4, "_device_of", lambda *t: -1)
    return fb4.PageTables(i32(n, max_pages), i32(n), i32(8), i32(1), 16)


def test_page_tables_are_checked_when_made(monkeypatch):
    tables(monkeypatch)
    for bad in ((i32(3), i32(3), i32(8), i32(1)), (i32(3, 4), i32(2), i32(8), i32(1)), (i32(3, 4), i32(3), i32(8), i32(2)),
                (i32(3, 4).long(), i32(3), i32(8), i32(1)), (i32(4, 3).t(), i32(3), i32(8), i32(1)), (i32(3, 4), i32(3), i32(16)[::2], i32(1))):
        with pytest.raises(ValueError):
            fb4.PageTables(*bad, 16)


def test_cache_plan_in_the_binding(monkeypatch):
    f = context(monkeypatch)
    pt = tables(monkeypatch)
    plan = f.cache_plan(pt, i32(3), 7, keep=i32(3))
    assert plan.q_start.shape == (4,) and plan.slot.shape == (7,) and plan.slot.dtype == torch.int64 and plan.pos.dtype == torch.int32
    assert [c[0] for c in f.calls] == ["fb4_cache_plan"]
    for new, rows, keep in ((i32(2), 7, None), (i32(3).long(), 7, None), (i32(6)[::2], 7, None), (i32(3), -1, None), (i32(3), 1 << 31, None),
                            (i32(3), 7, i32(4)), (i32(3), 7, i32(3).short())):
        with pytest.raises(ValueError):
            f.cache_plan(pt, new, rows, keep=keep)
    f.device = 0                                             # tensors of another device than the context's
    with pytest.raises(ValueError):
        f.cache_plan(pt, i32(3), 7)
    assert len(f.calls) == 1
