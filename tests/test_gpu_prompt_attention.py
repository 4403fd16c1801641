"""Attention over packed prompts, against the definition in 64 bits."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import attend, check

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def starts_of(lengths, at=0):
    out = [at]
    for n in lengths:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def seen_of(n, m, causal, window):
    i, j = torch.arange(n, device="cuda")[:, None] + (m - n), torch.arange(m, device="cuda")[None, :]
    seen = torch.ones(n, m, dtype=torch.bool, device="cuda")
    if causal:
        seen &= j <= i
    if window:
        seen &= j > i - window
    return seen


def definition(q, k, v, lq, lk, causal, window, scale, first_q=0, first_k=0):
    y, bound = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.full(q.shape, 1e-30, dtype=torch.float64, device="cuda")
    a, b = first_q, first_k
    for n, m in zip(lq, lk):
        if n and m:
            y[a:a + n], bound[a:a + n] = attend(q[a:a + n], k[b:b + m], v[b:b + m], seen_of(n, m, causal, window), scale)
        a, b = a + n, b + m
    return y, bound


def inputs(rows_q, rows_k, q_heads, kv_heads, dim, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda rows, heads: torch.randn(rows, heads, dim, generator=g, device="cuda").bfloat16()
    return make(rows_q, q_heads), make(rows_k, kv_heads), make(rows_k, kv_heads)


def case(lq, lk, q_heads, kv_heads, dim, causal=True, window=0, seed=0, scale=None):
    q, k, v = inputs(sum(lq), sum(lk), q_heads, kv_heads, dim, seed)
    y = nq.nq_prompt_attention(q, k, v, starts_of(lq), starts_of(lk), causal=causal, window=window, scale=scale)
    nq.nq_device_status()
    want, bound = definition(q, k, v, lq, lk, causal, window, dim ** -0.5 if scale is None else scale)
    check(y, want, bound)
    return q, k, v, y


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq", [[1], [128], [129], [256], [257], [384, 5], [1, 0, 127, 128, 700], [513, 511]])
def test_lengths(lq, causal, dim):
    case(lq, lq, 2, 1, dim, causal)


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (5, 5), (12, 4), (8, 1), (40, 2)])
def test_heads(q_heads, kv_heads):
    case([300, 77], [300, 77], q_heads, kv_heads, 64)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lq,lk", [([1], [1000]), ([130], [131]), ([5, 300], [260, 300]), ([200, 64, 300], [40, 0, 299]), ([257], [128]), ([600], [1]), ([128, 128], [384, 129])])
def test_prefixes_and_too_few_keys(lq, lk, dim):
    """More keys than queries: a prefix; fewer: the first rows of a causal sequence see nothing and are zero."""
    _, _, _, y = case(lq, lk, 4, 2, dim, True)
    a = 0
    for n, m in zip(lq, lk):
        assert bool((y[a: a + max(0, n - m)] == 0).all())
        a += n
    case(lq, lk, 4, 2, dim, False)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [1, 2, 100, 128, 129, 300, 100000])
def test_windows(window, causal):
    case([700, 3, 257], [700, 40, 200], 2, 1, 64, causal, window)


@pytest.mark.parametrize("scale", [1e-4, 0.3, 3.0])
def test_scales(scale):
    case([500], [500], 2, 2, 128, scale=scale)


@pytest.mark.parametrize("dim", [64, 128])
def test_long_sequence(dim):
    q, k, v, y = case([4100], [4100], 2, 1, dim)
    assert torch.equal(y, nq.nq_prompt_attention(q, k, v, starts_of([4100])))                  # bit for bit again


def test_many_sequences():
    g = torch.Generator().manual_seed(3)
    lq = [int(x) for x in torch.randint(0, 60, (900,), generator=g)]
    case(lq, lq, 2, 1, 64)


def test_scores_that_rise_along_the_keys():
    """The running maximum moves at every step, so all sums are rescaled."""
    n, dim = 900, 128
    q, k, v = inputs(n, n, 1, 1, dim)
    q = torch.ones_like(q)
    k = (k.float() * 0.01 + (torch.arange(n, device="cuda") / 16.0)[:, None, None]).bfloat16()
    y = nq.nq_prompt_attention(q, k, v, starts_of([n]), causal=False)
    want, bound = definition(q, k, v, [n], [n], False, 0, dim ** -0.5)
    check(y, want, bound)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 50), (False, 0)])
def test_hidden_keys_and_values_have_no_part(dim, bad, causal, window):
    """What is no number in another sequence, behind the last one or in a key or value that a row does not see."""
    lengths = [200, 300, 130]
    rows = sum(lengths) + 100
    q, k, v = inputs(rows, rows, 2, 1, dim)
    starts = starts_of(lengths, 50)
    for t in (q, k, v):
        t[:50], t[50 + sum(lengths):] = bad, bad
    bad_rows = [50 + 200 + 170, 50 + 200 + 255]                                               # in the second sequence
    clean = nq.nq_prompt_attention(q, k, v, starts, causal=causal, window=window)
    want, bound = definition(q, k, v, lengths, lengths, causal, window, dim ** -0.5, 50, 50)
    live = slice(50, 50 + sum(lengths))
    check(clean[live], want[live], bound[live])
    for which in (1, 2):
        args = [q, k.clone(), v.clone()]
        args[which][bad_rows] = bad
        y = nq.nq_prompt_attention(*args, starts, causal=causal, window=window)
        nq.nq_device_status()
        seen = seen_of(300, 300, causal, window)
        reached = torch.zeros(rows, dtype=torch.bool, device="cuda")
        reached[250:550] = seen[:, 170] | seen[:, 255]
        hidden = ~reached
        hidden[:50], hidden[50 + sum(lengths):] = False, False
        check(y[hidden], want[hidden], bound[hidden])                                        # weights that were summed by hand differ in their last bits
        if which == 2 or bad != bad:
            assert not torch.isfinite(y[reached]).all(-1).any()
        other = torch.cat([torch.arange(50, 250), torch.arange(550, 680)]).cuda()
        assert torch.equal(y[other], clean[other])


def test_infinite_value_that_some_rows_of_a_tile_see():
    n, dim = 100, 64
    q, k, v = inputs(n, n, 1, 1, dim)
    v[40, 0, 7] = float("inf")
    y = nq.nq_prompt_attention(q, k, v, starts_of([n]))
    assert torch.isfinite(y[:40]).all() and bool((y[40:, 0, 7] == float("inf")).all())
    others = [c for c in range(dim) if c != 7]
    w = v.clone()
    w[40, 0, 7] = 0.0
    want, bound = definition(q, k, w, [n], [n], True, 0, dim ** -0.5)
    check(y[..., others], want[..., others], bound[..., others])


def test_strides_and_rows_outside():
    lengths, dim = [140, 30], 128
    fused = torch.randn(200, 4 + 2 * 2, dim, device="cuda").bfloat16()
    q, k, v = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    starts = starts_of(lengths, 7)
    out = torch.full((200, 6, dim), 9.0, dtype=BF16, device="cuda")
    y = nq.nq_prompt_attention(q, k, v, starts, y_out=out[:, 1:5])
    want, bound = definition(q, k, v, lengths, lengths, True, 0, dim ** -0.5, 7, 7)
    check(y[7:177], want[7:177], bound[7:177])
    assert bool((out[:, 0] == 9).all()) and bool((out[:, 5] == 9).all()) and bool((out[:7] == 9).all()) and bool((out[177:] == 9).all())


def test_nothing_to_do():
    q, k, v = inputs(5, 0, 2, 1, 64)
    y = nq.nq_prompt_attention(q, k, v, starts_of([5]), starts_of([0]))
    assert bool((y == 0).all())
    assert nq.nq_prompt_attention(q[:0], k, v, starts_of([0])).shape == (0, 2, 64)
    out = torch.full_like(q, 3.0)
    nq.nq_prompt_attention(q, k, v, starts_of([]), y_out=out)
    assert bool((out == 3).all())


def test_starts_past_the_rows_are_held_back():
    q, k, v = inputs(100, 60, 1, 1, 64)
    starts_q, starts_k = torch.tensor([-5, 40, 1 << 30], dtype=torch.int32, device="cuda"), torch.tensor([0, 30, 2000], dtype=torch.int32, device="cuda")
    y = nq.nq_prompt_attention(q, k, v, starts_q, starts_k)
    want = nq.nq_prompt_attention(q, k, v, starts_of([40, 60]), starts_of([30, 30]))
    assert torch.equal(y, want)


def test_captured_call_follows_the_starts():
    q, k, v = inputs(1000, 1000, 4, 2, 128)
    starts = starts_of([1000])
    starts = torch.cat([starts, starts[-1:]])
    nq.nq_prompt_attention(q, k, v, starts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first = nq.nq_prompt_attention(q, k, v, starts)
        second = nq.nq_prompt_attention(first, k, v, starts)
    for cut in (1000, 1, 333, 0):
        starts.copy_(torch.tensor([0, cut, 1000], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = nq.nq_prompt_attention(q, k, v, starts)
        assert torch.equal(first, eager) and torch.equal(second, nq.nq_prompt_attention(eager, k, v, starts))


def test_two_streams_at_once():
    sets = [inputs(800, 800, 4, 2, 64, seed) for seed in (1, 2)]
    want = [nq.nq_prompt_attention(*s, starts_of([800])) for s in sets]
    starts = starts_of([800])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = nq.nq_prompt_attention(*sets[i], starts)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 70), (False, 200)])
@pytest.mark.parametrize("lq,lk", [([1], [1]), ([257, 128, 0, 129], [257, 128, 0, 129]), ([700], [900]), ([300, 40], [100, 290]), ([513], [513])])
def test_heads_that_do_not_pair(lq, lk, causal, window, dim):
    """An odd number of query heads a key head: a unit of work is 256 rows of one head."""
    case(lq, lk, 3, 1, dim, causal, window)
    case(lq, lk, 2, 2, dim, causal, window)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_hidden_values_where_heads_do_not_pair(bad):
    lengths = [300, 140]
    q, k, v = inputs(440, 440, 3, 3, 64)
    v[260], v[410] = bad, bad
    y = nq.nq_prompt_attention(q, k, v, starts_of(lengths))
    nq.nq_device_status()
    clean = v.clone()
    clean[260], clean[410] = 0.0, 0.0
    want, bound = definition(q, k, clean, lengths, lengths, True, 0, 0.125)
    for rows in (slice(0, 260), slice(300, 410)):
        check(y[rows], want[rows], bound[rows])
    assert not torch.isfinite(y[260:300]).all(-1).any() and not torch.isfinite(y[410:]).all(-1).any()
