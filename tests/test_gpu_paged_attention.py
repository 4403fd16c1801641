"""Attention of one new token over the paged cache, against the definition in 64 bits."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import attend, check, filled, sequence

pytestmark = pytest.mark.gpu
BF16, F8, I8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8


def definition(q, cache, table, lengths, window, scale):
    y, bound = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.full(q.shape, 1e-30, dtype=torch.float64, device="cuda")
    for i, n in enumerate(lengths):
        if n > 0:
            t = torch.arange(n, device="cuda")
            seen = (t >= n - window)[None] if window else torch.ones(1, n, dtype=torch.bool, device="cuda")
            y[i:i + 1], bound[i:i + 1] = attend(q[i:i + 1], sequence(cache, table[i], n, 0), sequence(cache, table[i], n, 1), seen, scale)
            if cache[3] is not None:
                bound[i] += held_as_f16(cache, table[i], n, seen[0], q.shape[1])
    return y, bound


def held_as_f16(cache, row, n, seen, heads):
    """What weights of 8-bit values lose beside bf16's half step.  A weight w (of the one at the running maximum, which is 1 and not above
    the largest) is held as f16(2^7 w vs / R), R the largest scale so far: under 2^-14 that is off by half of f16's least step, 2^-25, so
    the sum by at most 2^-25 2^-7 R sum |code|, and the sum of weights it is divided by is 1 at least."""
    codes = sequence((cache[0], cache[1], None, None), row, n, 1).abs()
    scales = sequence((cache[0], cache[3][..., None], None, None), row, n, 1)
    codes, scales = torch.where(seen[:, None, None], codes, 0.0), torch.where(seen[:, None, None], scales, 0.0)
    return (2.0 ** -32 * scales.abs().amax(0) * codes.sum(0)).repeat_interleave(heads // codes.shape[1], 0)


def case(lengths, group, kv_heads, dim, page, kind, window=0, seed=1, q_scale=1.0, scale=None):
    cache, table, device_lengths = filled(lengths, kv_heads, page, dim, kind, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 7)
    q = (q_scale * torch.randn(len(lengths), group * kv_heads, dim, generator=g, device="cuda")).bfloat16()
    y = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, device_lengths, window=window, scale=scale)
    want, bound = definition(q, cache, table, lengths, window, dim ** -0.5 if scale is None else scale)
    check(y, want, bound)
    for i, n in enumerate(lengths):
        if n <= 0:
            assert bool((y[i] == 0).all())
    return q, cache, table, device_lengths, y


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lengths,group,kv_heads,page", [
    ([1], 1, 1, 16), ([0, 5, 0, 16, 17, 15], 4, 2, 16), ([33, 1, 200], 8, 3, 48), ([700], 3, 1, 64), ([1501, 3], 16, 2, 16), ([90, 91], 5, 2, 32), ([130], 20, 1, 16),
    ([64, 80], 40, 2, 16)])
def test_lengths_and_groups(lengths, group, kv_heads, page, dim, kind):
    case(lengths, group, kv_heads, dim, page, kind)


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("lengths,window", [([40, 1, 300, 16], 1), ([40, 7, 300, 17], 16), ([100, 33], 17), ([1000, 31, 0], 250), ([50], 2000)])
def test_windows(lengths, window, kind):
    """What lies before the window is hidden, its not-a-numbers too."""
    cache, table, n = filled(lengths, 2, 16, 64, kind, 3)
    for i, length in enumerate(lengths):
        for t in range(0, max(0, length - window)):
            page = int(table[i, t // 16])
            for x, s in ((cache[0], cache[2]), (cache[1], cache[3])):
                if s is None:
                    x[page, :, t % 16] = float("nan")
                else:
                    s[page, :, t % 16] = float("nan")
    q = torch.randn(len(lengths), 8, 64, device="cuda").bfloat16()
    y = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n, window=window)
    want, bound = definition(q, cache, table, lengths, window, 0.125)
    check(y, want, bound)


@pytest.mark.parametrize("kind", [BF16, F8, I8])
def test_long_sequences_are_split_and_joined(kind):
    q, cache, table, n, y = case([20011, 3, 9000], 4, 2, 128, 16, kind)
    assert torch.equal(y, nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n))                        # bit for bit again


@pytest.mark.parametrize("kind", [BF16, F8])
def test_many_short_sequences(kind):
    g = torch.Generator().manual_seed(5)
    case([int(v) for v in torch.randint(0, 90, (700,), generator=g)], 2, 3, 64, 16, kind)


def test_more_sequences_than_chunks_and_empty_ones_between():
    lengths = [0] * 3000
    lengths[17], lengths[1500], lengths[2999] = 400, 33, 1
    case(lengths, 2, 1, 64, 16, BF16)
    case([0] * 5, 2, 1, 64, 16, F8)


@pytest.mark.parametrize("kind", [BF16, F8, I8])
def test_large_and_small_scores(kind):
    case([513], 8, 1, 128, 16, kind, q_scale=30.0)                           # one token takes nearly all
    case([513], 8, 1, 128, 16, kind, q_scale=1e-30)                          # all alike; f16 would lose such queries
    case([77], 2, 1, 64, 16, kind, q_scale=1e4, scale=1e-6)


@pytest.mark.parametrize("kind", [F8, I8])
def test_values_of_very_different_sizes(kind):
    cache, table, n = filled([300], 1, 16, 64, kind, 9)
    cache[3].mul_(torch.exp(20 * torch.randn(cache[3].shape, device="cuda")))
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    y = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n)
    want, bound = definition(q, cache, table, [300], 0, 0.125)
    check(y, want, bound)


@pytest.mark.parametrize("kind", [BF16, F8, I8])
def test_pages_outside_the_cache_are_hidden(kind):
    cache, table, n = filled([100, 40, 20], 2, 16, 64, kind, 4)
    pages = cache[0].shape[0]
    q = torch.randn(3, 4, 64, device="cuda").bfloat16()
    gone = table.clone()
    gone[0, 2], gone[0, 6], gone[1, 0], gone[2, 0], gone[2, 1] = -1, pages, 1 << 30, -(1 << 31), pages + 5
    y = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), gone, n)
    for i, (length, hidden) in enumerate([(100, (2, 6)), (40, (0,)), (20, (0, 1))]):
        t = torch.arange(length, device="cuda") // 16
        seen = torch.ones(length, dtype=torch.bool, device="cuda")
        for h in hidden:
            seen &= t != h
        if not bool(seen.any()):
            assert bool((y[i] == 0).all())
            continue
        want, bound = attend(q[i:i + 1], sequence(cache, table[i], length, 0), sequence(cache, table[i], length, 1), seen[None], 0.125)
        if cache[3] is not None:
            bound[0] += held_as_f16(cache, table[i], length, seen, 4)
        check(y[i:i + 1], want, bound)


def test_length_past_the_table_is_what_the_table_holds():
    cache, table, n = filled([64, 30], 1, 16, 64, BF16, 4)
    q = torch.randn(2, 2, 64, device="cuda").bfloat16()
    long = torch.tensor([1 << 30, 30], dtype=torch.int32, device="cuda")
    assert torch.equal(nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, long), nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n))


@pytest.mark.parametrize("kind", [BF16, F8, I8])
def test_infinities_and_no_numbers_that_are_seen(kind):
    """A key, value or query that is no number reaches its own sequence's result, and no other's."""
    cache, table, n = filled([40, 40, 40], 1, 16, 64, kind, 6)
    q = torch.randn(3, 2, 64, device="cuda").bfloat16()
    clean = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n)
    page = int(table[1, 1])
    for which in (0, 1):
        for bad in (float("nan"), float("inf")):
            c = [None if t is None else t.clone() for t in cache]
            if kind is BF16:
                c[which][page, 0, 3] = bad
            else:
                c[2 + which][page, 0, 3] = bad
            y = nq.nq_paged_attention(q, nq.nq_kv_pages(*c), table, n)
            assert torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2])
            assert not torch.isfinite(y[1]).all()
    bad_q = q.clone()
    bad_q[1, 1] = float("nan")
    y = nq.nq_paged_attention(bad_q, nq.nq_kv_pages(*cache), table, n)
    assert torch.isnan(y[1, 1]).all() and torch.equal(y[0], clean[0]) and torch.equal(y[1, 0], clean[1, 0])


def test_strides_outputs_and_workspaces():
    cache, table, n = filled([50, 20, 3], 2, 16, 64, F8, 8)
    c = nq.nq_kv_pages(*cache)
    wide = torch.randn(3, 9, 64, device="cuda").bfloat16()
    q = wide[:, 2:6]
    plain = nq.nq_paged_attention(q.contiguous(), c, table, n)
    out = torch.full((3, 7, 64), 5.0, dtype=BF16, device="cuda")
    space = torch.full((nq.nq_paged_attention_workspace_bytes(c, 4, 3, table.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    pitched = torch.full((3, table.shape[1] + 5), 77, dtype=torch.int32, device="cuda")
    pitched[:, : table.shape[1]] = table
    got = nq.nq_paged_attention(q, c, pitched[:, : table.shape[1]], n, y_out=out[:, 1:5], workspace=space)
    assert torch.equal(got, plain) and bool((out[:, 0] == 5).all()) and bool((out[:, 5:] == 5).all())


def test_captured_call_follows_lengths_and_tables():
    cache, table, n = filled([3000, 100], 2, 16, 128, F8, 8, hole=0.0)
    c = nq.nq_kv_pages(*cache)
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    nq.nq_paged_attention(q, c, table, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = nq.nq_paged_attention(q, c, table, n)
        second = nq.nq_paged_attention(first, c, table, n)
    for lengths in ([3000, 100], [1, 0], [2999, 101 - 5]):
        n.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = nq.nq_paged_attention(q, c, table, n)
        assert torch.equal(first, eager) and torch.equal(second, nq.nq_paged_attention(eager, c, table, n))


def test_two_streams_at_once():
    cache, table, n = filled([5000, 2000], 2, 16, 128, BF16, 8)
    c = nq.nq_kv_pages(*cache)
    qs = [torch.randn(2, 8, 128, device="cuda").bfloat16() for _ in range(2)]
    want = [nq.nq_paged_attention(q, c, table, n) for q in qs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = nq.nq_paged_attention(qs[i], c, table, n)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", [F8, I8])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_key_of_infinite_scale_is_no_number_whatever_its_score(kind, sign):
    cache, table, n = filled([20], 1, 16, 64, kind, 2)
    q = torch.full((1, 4, 64), sign, device="cuda").bfloat16()
    page = int(table[0, 0])
    cache[0][page, 0, 5] = torch.ones(64, device="cuda").to(kind)
    cache[2][page, 0, 5] = float("inf")
    assert torch.isnan(nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n)).all()


@pytest.mark.parametrize("kind", [BF16, F8])
def test_calls_one_behind_another_share_nothing(kind):
    """Many calls of different sizes in a row, each launched while the one before still runs."""
    made = [filled(lengths, 2, 16, 64, kind, seed) for seed, lengths in enumerate([[3000, 5], [1] * 300, [0, 700, 0], [17]])]
    qs = [torch.randn(len(m[2]), 8, 64, device="cuda").bfloat16() for m in made]
    call = lambda i: nq.nq_paged_attention(qs[i], nq.nq_kv_pages(*made[i][0]), made[i][1], made[i][2])
    want = []
    for i in range(4):
        want.append(call(i))
        torch.cuda.synchronize()
    for _ in range(30):
        got = [call(i) for i in (0, 1, 2, 3, 1, 0)]
    torch.cuda.synchronize()
    for i, y in zip((0, 1, 2, 3, 1, 0), got):
        assert torch.equal(y, want[i])


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("lengths,group,dim,window", [([40007], 4, 128, 0), ([40007, 60], 16, 64, 0), ([9001, 1, 700], 40, 128, 0), ([50000], 3, 128, 39001)])
def test_one_head_is_split_over_all_thread_blocks(lengths, group, dim, window, kind):
    """More parts of a head than the joining kernel has threads; a group of several blocks of heads."""
    q, cache, table, n, y = case(lengths, group, 1, dim, 16, kind, window=window)
    assert torch.equal(y, nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n, window=window))
