"""Tokens past the last position of a served stack are refused on the host: their keys would be NaN and stay in the cache."""
import pytest
import torch

from paper_2506_17870_b200.attention import AttentionBlock, DecoderStack, PageTable, rotary_angles


def test_a_page_table_ends_at_its_positions():
    t = PageTable(10, 16, device="cpu", positions=40)
    a, b = t.add(), t.add()
    assert t.extend([a, b], [39, 40]).longest == 40
    free = t.free_pages
    with pytest.raises(RuntimeError, match="41 tokens of a sequence, there are 40 positions"):
        t.extend([a, b], [1, 1])
    assert t.length(a) == 39 and t.length(b) == 40 and t.free_pages == free           # nothing has changed
    assert t.extend([a], [1]).longest == 40 and t.extend([b], [0]).longest == 40
    t.drop(b)
    assert t.extend([t.add()], [17]).longest == 17
    assert PageTable(10, 16, device="cpu").extend([], []).longest == 0
    with pytest.raises(ValueError):
        PageTable(10, 16, device="cpu", positions=-1)


def test_a_stacks_table_has_its_positions(monkeypatch):
    monkeypatch.setattr(AttentionBlock, "cache", lambda *_: None)
    table = DecoderStack(1, 64, 64, 1, 1, 64, positions=33, device="cpu").cache(8, 16)
    a = table.add()
    table.extend([a], [33])
    with pytest.raises(RuntimeError, match="positions"):
        table.extend([a], [1])


def test_a_batch_longer_than_the_angles_is_not_served():
    t = PageTable(10, 16, device="cpu")
    a = t.add()
    t.extend([a], [64])
    block = AttentionBlock(64, 1, 1, 64, device="cpu")
    angles = rotary_angles(64, 64, device="cpu")
    with pytest.raises(ValueError, match="65 tokens of a sequence, angles of 64 positions"):
        block.serve(torch.zeros(1, 64), torch.zeros(1, 1), t.extend([a], [1]), angles)
