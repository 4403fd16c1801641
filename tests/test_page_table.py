"""Who holds which pages of a cache: host bookkeeping, no GPU."""
import pytest
import torch

from paper_2506_17870_b200.attention import PageTable, rotary_angles


def test_tokens_go_to_the_pages_that_are_listed():
    t = PageTable(10, 16, device="cpu")
    a, b = t.add(), t.add()
    x = t.extend([a, b], [20, 3])
    assert x.fresh and not x.single and x.starts.tolist() == [0, 20, 23] and x.starts_all.tolist() == [0, 20, 23] and x.lengths.tolist() == [20, 3] and x.rows_all == 23
    assert x.positions.tolist() == list(range(20)) + list(range(3)) and x.table.shape == (2, 2) and t.free_pages == 7
    for row, n, at in ((0, 20, 0), (1, 3, 20)):
        for i in range(n):
            assert x.slots[at + i] == x.table[row, i // 16] * 16 + i % 16
    assert x.table[1, 1] == -1 and len(set(x.slots.tolist())) == 23
    y = t.extend([b, a], [1, 1])
    assert y.single and not y.fresh and y.positions.tolist() == [3, 20] and y.lengths.tolist() == [4, 21] and y.starts_all.tolist() == [0, 4, 25]
    assert y.slots.tolist() == [int(x.table[1, 0]) * 16 + 3, int(x.table[0, 1]) * 16 + 4]
    z = t.extend([a, b], [0, 29])
    assert z.starts.tolist() == [0, 0, 29] and z.lengths.tolist() == [21, 33] and t.free_pages == 5 and t.length(b) == 33
    assert all(v.dtype == torch.int32 for v in z[:6])


def test_pages_come_back():
    t = PageTable(3, 16, device="cpu")
    a, b = t.add(), t.add()
    t.extend([a, b], [17, 16])
    with pytest.raises(RuntimeError, match="1 pages needed, 0 free"):
        t.extend([b], [1])
    assert t.length(b) == 16
    t.drop(a)
    assert t.free_pages == 2
    t.extend([b], [32])
    assert t.free_pages == 0
    with pytest.raises(KeyError):
        t.length(a)


def test_refusals():
    t = PageTable(3, 16, device="cpu")
    a = t.add()
    for sequences, counts in (([a], [1, 2]), ([a, a], [1, 1]), ([a], [-1])):
        with pytest.raises(ValueError):
            t.extend(sequences, counts)
    with pytest.raises(ValueError):
        PageTable(-1, 16)
    assert t.free_pages == 3


def test_angles_are_those_of_64_bits():
    a = rotary_angles(1 << 17, 64, device="cpu")
    at = (1 << 17) - 1
    want = torch.tensor([at * 10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    assert a.shape == (1 << 17, 64) and float((a[at] - torch.cat([want.cos(), want.sin()])).abs().max()) <= 2.0 ** -24 + 2.0 ** -30
