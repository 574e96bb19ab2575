"""Attention side of the binding on the CPU: what it refuses before anything reaches the library.  The context here has no device: its
calls are recorded instead of made."""
from types import SimpleNamespace

import pytest
import torch

from paper_2603_02883_b200 import fb4


def context(monkeypatch, block_size=32):
    f = fb4.Fb4.__new__(fb4.Fb4)
    f.ctx, f.device, f.block_size, f.calls = None, -1, block_size, []         # -1 is the device index of CPU tensors
    monkeypatch.setattr(fb4.Fb4, "_call", lambda self, where, *args: self.calls.append((where, args)))
    return f


def cpu_cache(n_pages=3, page=16, heads=2, D=64):
    t = SimpleNamespace(k_codes=torch.zeros(n_pages, heads, page, D // 2, dtype=torch.uint8), k_meta=torch.zeros(n_pages, heads, page, D // 32, dtype=torch.int16),
                        v_codes=torch.zeros(n_pages, heads, page, D // 2, dtype=torch.uint8), v_meta=torch.zeros(n_pages, heads, page, D // 32, dtype=torch.int16))
    t._c = fb4.Fb4Cache(t.k_codes.data_ptr(), t.k_meta.data_ptr(), t.v_codes.data_ptr(), t.v_meta.data_ptr(), n_pages, page, heads, D), -1
    return t


def test_cache_values_needs_block_size_32(monkeypatch):
    """a context of block size 16 would read two metadata words where the cache has one, past the end of the array"""
    f = context(monkeypatch, block_size=16)
    with pytest.raises(fb4.Fb4Error) as e:
        f.cache_values(cpu_cache())
    assert e.value.code == fb4.ERR_INVALID_ARG and not f.calls
    g = context(monkeypatch)
    k, v = g.cache_values(cpu_cache(), torch.bfloat16)
    assert k.shape == v.shape == (3, 2, 16, 64) and [c[0] for c in g.calls] == ["fb4_dequantize"] * 2


def test_an_output_type_that_is_none_of_the_three_is_refused_first(monkeypatch):
    f = context(monkeypatch)
    made = []
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda self, *a, **k: made.append(a))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32)  # noqa: E731
    for bad in (torch.float64, torch.int8, torch.float8_e4m3fn, None, "bf16"):
        with pytest.raises(ValueError):
            f.cache_values(cpu_cache(), bad)
        with pytest.raises(ValueError):
            f.cache_attention(torch.zeros(1, 4, 64, dtype=torch.bfloat16), cpu_cache(), i32(0)[None], i32(1), i32(0, 1), 1, 1, dtype=bad)
    assert not f.calls and not made
