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
  if (plan(w, 4, 16, w, w, 2, w, 8, w, -1, w, slot, w) != FB4_ERR_SHAPE || plan(w, 4, 16, w, w, 2, w, 8, w, (1LL << 30) + 1, w, slot, w) != FB4_ERR_SHAPE) return 8;
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
    for new, rows, keep in ((i32(2), 7, None), (i32(3).long(), 7, None), (i32(6)[::2], 7, None), (i32(3), -1, None), (i32(3), (1 << 30) + 1, None),
                            (i32(3), 7, i32(4)), (i32(3), 7, i32(3).short())):
        with pytest.raises(ValueError):
            f.cache_plan(pt, new, rows, keep=keep)
    f.device = 0                                             # tensors of another device than the context's
    with pytest.raises(ValueError):
        f.cache_plan(pt, i32(3), 7)
    assert len(f.calls) == 1


CACHE8 = r"""
  fb4_cache8 c8;
  memset(&c8, 0, sizeof c8);
  c8.k = c8.v = c8.k_scale = c8.v_scale = room;
  c8.n_pages = 4;
  c8.page_tokens = 16;
  c8.n_heads = 2;
  c8.head_dim = 64;
  struct Args {
    fb4_cache8 c;
    const int32_t *table, *kv, *start;
    int max_pages, n, max_q;
    const void *k, *v, *q, *gain;
    int64_t k_ld, v_ld, q_ld, T, out_ld;
    float eps;
    int q_heads;
    void* out;
  };
  const Args ok{c8, lens, lens, lens, 4, 2, 8, room, room, room, room, 128, 128, 64, 10, 64, 1e-6f, 1, room + 4096};
  auto append = [&](const Args& a) {
    return fb4_cache8_append(&ctx, &a.c, a.table, a.max_pages, a.kv, a.start, a.n, a.max_q, a.k, a.k_ld, a.v, a.v_ld, a.T, a.gain, a.eps, 0, a.q, a.q_heads,
                             a.q_ld, a.gain, a.out, a.out_ld, 0);
  };
  auto attend = [&](const Args& a, float scale, int causal, int window, int dtype, int max_kv) {
    return fb4_cache8_attention(&ctx, a.q, 128, 2, a.T, &a.c, a.table, a.max_pages, a.kv, a.start, a.n, a.max_q, max_kv, scale, causal, window, a.out, 128, dtype,
                                0, 0, 0, 0);
  };
  auto both = [&](const Args& a, int code) { return append(a) == code && attend(a, 0.1f, 1, 0, 1, 64) == code && fb4_cache8_values(&ctx, &a.c, room, room, 0, 0) == code; };
  ctx.attend_error = cudaErrorInvalidConfiguration;
  if (attend(ok, 0.1f, 1, 0, 1, 64) != FB4_ERR_CUDA || fb4_last_cuda_error() != (int)cudaErrorInvalidConfiguration) return 1;
  Args a = ok;
  for (int page : {0, 8, 24, 8192}) { a.c.page_tokens = page; if (!both(a, FB4_ERR_SHAPE)) return 2; }
  for (int D : {0, 16, 48, 288}) { a = ok; a.c.head_dim = D; if (!both(a, FB4_ERR_SHAPE)) return 3; }
  for (int h : {0, 1025}) { a = ok; a.c.n_heads = h; if (!both(a, FB4_ERR_SHAPE)) return 4; }
  for (int64_t n : {0LL, -1LL, 1LL << 37}) { a = ok; a.c.n_pages = n; if (!both(a, FB4_ERR_SHAPE)) return 5; }
  a = ok; a.c.k = 0; if (!both(a, FB4_ERR_INVALID_ARG)) return 6;
  a = ok; a.c.v_scale = 0; if (!both(a, FB4_ERR_INVALID_ARG)) return 7;
  a = ok; a.c.v = room + 8; if (!both(a, FB4_ERR_ALIGN)) return 8;
  a = ok; a.T = -1; if (append(a) != FB4_ERR_SHAPE) return 9;
  a = ok; a.n = -1; if (append(a) != FB4_ERR_SHAPE) return 10;
  a = ok; a.n = (1 << 28) + 1; if (append(a) != FB4_ERR_SHAPE) return 11;
  a = ok; a.max_q = -1; if (append(a) != FB4_ERR_SHAPE) return 12;
  a = ok; a.table = 0; if (append(a) != FB4_ERR_INVALID_ARG) return 13;
  a = ok; a.kv = 0; if (append(a) != FB4_ERR_INVALID_ARG) return 14;
  a = ok; a.k = 0; if (append(a) != FB4_ERR_INVALID_ARG) return 15;
  a = ok; a.k_ld = 120; if (append(a) != FB4_ERR_SHAPE) return 16;
  a = ok; a.v_ld = 132; if (append(a) != FB4_ERR_ALIGN) return 17;
  a = ok; a.q = 0; if (append(a) != FB4_ERR_INVALID_ARG) return 18;
  a = ok; a.out = room + 8; if (append(a) != FB4_ERR_ALIGN) return 19;
  a = ok; a.gain = room + 2; if (append(a) != FB4_ERR_ALIGN) return 20;
  a = ok; a.eps = -1.0f; if (append(a) != FB4_ERR_INVALID_ARG) return 21;
  a = ok; a.q_heads = 1025; if (append(a) != FB4_ERR_SHAPE) return 22;
  a = ok; a.q = a.out; a.q_ld = 72; if (append(a) != FB4_ERR_INVALID_ARG) return 23;                     // in place with another stride
  a = ok; a.start = reinterpret_cast<const int32_t*>(room + 2); if (append(a) != FB4_ERR_ALIGN) return 24;
  for (int none = 0; none < 4; ++none) {                                                               // nothing to do
    a = ok;
    (none == 0 ? a.n : none == 1 ? a.max_q : a.max_pages) = 0;
    if (none == 3) a.T = 0;
    if (append(a) != FB4_OK) return 25;
  }
  if (fb4_cache8_values(&ctx, &c8, 0, room, 0, 0) != FB4_ERR_INVALID_ARG || fb4_cache8_values(&ctx, &c8, room, room + 8, 0, 0) != FB4_ERR_ALIGN) return 26;
  if (fb4_cache8_values(&ctx, &c8, room, room, 3, 0) != FB4_ERR_INVALID_ARG) return 27;
  if (attend(ok, 0.1f, 2, 0, 1, 64) != FB4_ERR_INVALID_ARG || attend(ok, 0.1f, 1, -1, 1, 64) != FB4_ERR_INVALID_ARG || attend(ok, 0.1f, 1, 0, 3, 64) != FB4_ERR_INVALID_ARG) return 28;
  if (attend(ok, 0x1p61f, 1, 0, 1, 64) != FB4_ERR_INVALID_ARG || attend(ok, 0.0f / 0.0f, 1, 0, 1, 64) != FB4_ERR_INVALID_ARG) return 29;
  if (attend(ok, 0.1f, 1, 0, 1, (1 << 30) + 1) != FB4_ERR_SHAPE) return 30;
  if (fb4_cache8_attention_workspace(&ctx, 3, 2, 64, 1, 1, 1, 0) != -1 || fb4_cache8_attention_workspace(0, 2, 2, 64, 1, 1, 1, 0) != -1) return 31;
  if (fb4_cache8_append(0, &c8, lens, 4, lens, lens, 2, 8, room, 128, room, 128, 10, 0, 0.0f, 0, 0, 0, 0, 0, 0, 0, 0) != FB4_ERR_INVALID_ARG) return 32;
  if (ctx.launches != 0) return 33;
  puts("ok");
  return 0;
}
"""


def test_cache8_refusals(tmp_path):
    run(tmp_path, CACHE8)


def cache8(monkeypatch, n=4, heads=2, page=16, D=64):
    monkeypatch.setattr(fb4, "_device_of", lambda *t: -1)
    codes, scale = torch.zeros(n, heads, page, D, dtype=torch.uint8), torch.zeros(n, heads, page // 16, dtype=torch.uint8)
    return fb4.Cache8(codes, scale, codes.clone(), scale.clone())


def test_cache8_in_the_binding(monkeypatch):
    f = context(monkeypatch)
    c = cache8(monkeypatch)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    for bad in ((u8(4, 2, 16), u8(4, 2, 1)), (u8(4, 2, 16, 64).short(), u8(4, 2, 1)), (u8(4, 2, 16, 64), u8(4, 2, 2)), (u8(4, 2, 64, 16).transpose(2, 3), u8(4, 2, 1))):
        with pytest.raises(ValueError):
            fb4.Cache8(*bad, u8(4, 2, 16, 64), u8(4, 2, 1))
    kv = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    ok = (c, kv, kv, i32(3, 4), i32(3), i32(4), 2)
    assert f.cache8_append(*ok) is None and f.cache8_append(*ok, q=torch.zeros(5, 6, 64, dtype=torch.bfloat16)).shape == (5, 6, 64)
    n = len(f.calls)
    swap = lambda at, x: tuple(x if i == at else y for i, y in enumerate(ok))  # noqa: E731
    for args, more in ((swap(1, kv[:, :1]), {}), (swap(1, kv.float()), {}), (swap(2, kv[:4]), {}), (swap(3, i32(2, 4)), {}), (swap(4, i32(3).long()), {}), (swap(5, i32(3)), {}),
                       (swap(6, 1 << 31), {}), (swap(6, -1), {}), (ok, dict(q=kv[:4])), (ok, dict(k_gain=kv[0, 0, :32])), (ok, dict(q=kv, q_gain=kv[0, 0].float()))):
        with pytest.raises(ValueError):
            f.cache8_append(*args, **more)
    for bad in (torch.float64, torch.int8, None):
        with pytest.raises(ValueError):
            f.cache8_values(c, bad)
        with pytest.raises(ValueError):
            f.cache8_attention(kv, c, i32(3, 4), i32(3), i32(4), 2, 16, dtype=bad)
    with pytest.raises(ValueError):
        f.cache8_attention(kv[..., :32], c, i32(3, 4), i32(3), i32(4), 2, 16)
    assert len(f.calls) == n


LINEAR = r"""
  const uint16_t* meta = reinterpret_cast<const uint16_t*>(room);
  ctx.linear_error = cudaErrorInvalidConfiguration;
  auto linear = [&](const void* x, int64_t T, int64_t K, int64_t ld, const uint8_t* codes, const uint16_t* m, int64_t N, const void* bias, void* out, int64_t out_ld, int dtype) {
    return fb4_linear(&ctx, x, T, K, ld, codes, m, N, bias, out, out_ld, dtype, 0);
  };
  if (linear(room, 4, 64, 64, room, meta, 10, room, room, 10, 1) != FB4_ERR_CUDA || fb4_last_cuda_error() != (int)cudaErrorInvalidConfiguration) return 1;
  for (int64_t K : {0, 16, 33, 48, -32}) if (linear(room, 4, K, 64, room, meta, 10, room, room, 10, 1) != FB4_ERR_SHAPE) return 2;
  if (linear(room, 4, 64, 56, room, meta, 10, 0, room, 10, 1) != FB4_ERR_SHAPE || linear(room, 4, 64, 64, room, meta, 10, 0, room, 9, 1) != FB4_ERR_SHAPE) return 3;
  if (linear(room, -1, 64, 64, room, meta, 10, 0, room, 10, 1) != FB4_ERR_SHAPE || linear(room, (1 << 22) + 1, 64, 64, room, meta, 10, 0, room, 10, 1) != FB4_ERR_SHAPE) return 4;
  if (linear(room, 4, 64, 64, room, meta, -1, 0, room, 10, 1) != FB4_ERR_SHAPE || linear(room, 4, 64, 64, room, meta, 1LL << 31, 0, room, 1LL << 31, 1) != FB4_ERR_SHAPE) return 5;
  if (linear(0, 4, 64, 64, room, meta, 10, 0, room, 10, 1) != FB4_ERR_INVALID_ARG || linear(room, 4, 64, 64, 0, meta, 10, 0, room, 10, 1) != FB4_ERR_INVALID_ARG) return 6;
  if (linear(room, 4, 64, 64, room, 0, 10, 0, room, 10, 1) != FB4_ERR_INVALID_ARG || linear(room, 4, 64, 64, room, meta, 10, 0, 0, 10, 1) != FB4_ERR_INVALID_ARG) return 7;
  if (linear(room, 4, 64, 64, room, meta, 10, 0, room, 10, 3) != FB4_ERR_INVALID_ARG || linear(room, 4, 64, 64, room, meta, 10, 0, room, 10, -1) != FB4_ERR_INVALID_ARG) return 8;
  if (linear(room + 8, 4, 64, 64, room, meta, 10, 0, room, 10, 1) != FB4_ERR_ALIGN || linear(room, 4, 64, 68, room, meta, 10, 0, room, 10, 1) != FB4_ERR_ALIGN) return 9;
  if (linear(room, 4, 64, 64, room + 8, meta, 10, 0, room, 10, 1) != FB4_ERR_ALIGN || linear(room, 4, 64, 64, room, meta + 1, 10, 0, room, 10, 1) != FB4_ERR_ALIGN) return 10;
  if (linear(room, 4, 64, 64, room, meta, 10, room + 1, room, 10, 1) != FB4_ERR_ALIGN || linear(room, 4, 64, 64, room, meta, 10, 0, room + 4, 10, 1) != FB4_ERR_ALIGN) return 11;
  if (linear(0, 0, 64, 64, 0, 0, 10, 0, 0, 10, 1) != FB4_OK || linear(0, 4, 64, 64, 0, 0, 0, 0, 0, 10, 1) != FB4_OK) return 12;
  ctx.cfg.block_size = 16;
  if (linear(room, 4, 64, 64, room, meta, 10, 0, room, 10, 1) != FB4_ERR_INVALID_ARG) return 13;
  if (fb4_linear(0, room, 4, 64, 64, room, meta, 10, 0, room, 10, 1, 0) != FB4_ERR_INVALID_ARG || ctx.launches != 0) return 14;
  puts("ok");
  return 0;
}
"""


def test_linear_refusals(tmp_path):
    run(tmp_path, LINEAR)


def test_linear_in_the_binding(monkeypatch):
    f = context(monkeypatch)
    w = fb4.Quantized(torch.zeros(10, 32, dtype=torch.uint8), torch.zeros(10, 2, dtype=torch.int16))
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    assert f.linear(x, w).shape == (4, 10) and f.linear(x, w, bias=x[0, :10], dtype=torch.float32).dtype == torch.float32 and len(f.calls) == 2
    swap = lambda **k: fb4.Quantized(**{**dict(codes=w.codes, meta=w.meta), **k})  # noqa: E731
    for bad in ((x.float(), w), (x[0], w), (x[:, :32], w), (x.t().contiguous().t(), w), (x, swap(codes=w.codes.short())), (x, swap(meta=w.meta[:9])), (x, swap(meta=w.meta.int())),
                (x, swap(codes=torch.zeros(32, 10, dtype=torch.uint8).t())), (x, w, x[0, :9]), (x, w, x[0, :10].float()), (x, w, x[:, 0]), (x, w, None, torch.float64),
                (x, swap(salient_idx=torch.zeros(1, dtype=torch.int32), res_codes=w.codes[:1], res_meta=w.meta[:1]))):
        with pytest.raises(ValueError):
            f.linear(*bad)
    assert len(f.calls) == 2
