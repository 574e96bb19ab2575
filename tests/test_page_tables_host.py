"""Sizes of page tables that 32 bits cannot hold are refused by the binding, which would pass them on cut off: 2^32 + 16 tokens as 16."""
import pytest
import torch

from paper_2603_02883_b200 import fb4
from test_attention_binding import context


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("tokens", [(1 << 32) + 16, 1 << 31, -1, -(1 << 32) + 16])
def test_page_tokens(monkeypatch, tokens):
    monkeypatch.setattr(fb4, "_device_of", lambda *t: -1)
    fb4.PageTables(i32(3, 4), i32(3), i32(8), i32(1), 16)
    with pytest.raises(ValueError):
        fb4.PageTables(i32(3, 4), i32(3), i32(8), i32(1), tokens)


@pytest.mark.parametrize("which", ["sequences", "pages of a sequence", "list"])
def test_sizes_of_the_tables(monkeypatch, which):
    """tensors without memory"""
    monkeypatch.setattr(fb4, "_device_of", lambda *t: -1)
    far = (1 << 32) + 8
    meta = lambda *s: torch.empty(s, dtype=torch.int32, device="meta")  # noqa: E731
    args = [i32(3, 4), i32(3), i32(8), i32(1)]
    if which == "sequences":
        args[:2] = meta(far, 0), meta(far)
    elif which == "pages of a sequence":
        args[0] = meta(3, far)
    else:
        args[2] = meta(far)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda self: 0)
    with pytest.raises(ValueError):
        fb4.PageTables(*args, 16)


def test_a_page_table_wider_than_32_bits(monkeypatch):
    """as the appends and the attention read it"""
    f = context(monkeypatch)
    with pytest.raises(ValueError):
        f._sequences(torch.empty((3, (1 << 32) + 8), dtype=torch.int32, device="meta"), i32(3), i32(4))
    assert f._sequences(i32(3, 8), i32(3), i32(4)) == 3
