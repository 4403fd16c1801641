"""Attention of new tokens over 8-bit caches whose values' scales differ widely, against the definition in 64 bits."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import MOST, attend, check, filled, sequence

pytestmark = pytest.mark.gpu
F8, I8 = torch.float8_e4m3fn, torch.int8


def token_definition(q, cache, table, lengths, window, scale):
    """The attention of new tokens in 64 bits and a bound: attend()'s, and what weights of 8-bit values lose as f16.  A weight times its
    value's scale, w vs, is held as f16 in units of no more than 2^-7 of the largest such product of the row, P: under 2^-14 that is off by half of
    f16's least step, 2^-25, so the sum of w vs code by at most 2^-32 P sum |code|."""
    y, bound = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.full(q.shape, 1e-30, dtype=torch.float64, device="cuda")
    for i, n in enumerate(lengths):
        if n == 0:
            continue
        t = torch.arange(n, device="cuda")
        seen = (t >= n - window)[None] if window else torch.ones(1, n, dtype=torch.bool, device="cuda")
        k, v = sequence(cache, table[i], n, 0), sequence(cache, table[i], n, 1)
        y[i:i + 1], bound[i:i + 1] = attend(q[i:i + 1], k, v, seen, scale)
        codes = sequence((cache[0], cache[1], None, None), table[i], n, 1).abs()
        scales = sequence((cache[0], cache[3][..., None], None, None), table[i], n, 1)[..., 0].abs()
        group = q.shape[1] // k.shape[1]
        for h in range(q.shape[1]):
            s = (k[:, h // group] @ q[i, h].double() * scale).masked_fill(~seen[0], -float("inf"))
            product = torch.where(seen[0], torch.softmax(s, 0) * scales[:, h // group], 0.0).max()
            bound[i, h] += 2.0 ** -32 * product * torch.where(seen[0][:, None], codes[:, h // group], 0.0).sum(0)
    return y, bound


@pytest.mark.parametrize("kind", [F8, I8])
@pytest.mark.parametrize("dim,group", [(64, 4), (128, 3), (64, 16), (128, 16)])
@pytest.mark.parametrize("length,at", [(50, 0), (50, 17), (50, 49), (3000, 0), (3000, 2999), (20011, 9000)])
@pytest.mark.parametrize("larger", [20, 33, 60])
def test_a_large_value_of_no_weight_takes_nothing_from_the_others(larger, length, at, dim, group, kind):
    """One token's score is 40 below the others' and its value's scale far above theirs: the tokens that hold the weight stay as precise as they are."""
    cache, table, n = filled([length], 2, 16, dim, kind, length + at)
    g = torch.Generator(device="cuda").manual_seed(at)
    score = -torch.rand(length, 2, generator=g, device="cuda")
    score[at] = -40.0
    t = torch.arange(length, device="cuda")
    page, place = table[0, t // 16].long(), t % 16
    codes = torch.full((length, 2, dim), float(MOST[kind]), device="cuda") * score.sign()[..., None]
    cache[0].view(torch.uint8)[page, :, place] = codes.to(kind).view(torch.uint8)
    cache[2][page, :, place] = score.abs() / (MOST[kind] * dim ** 0.5)
    cache[3][page[at], :, place[at]] *= 2.0 ** larger
    q = torch.ones(1, 2 * group, dim, device="cuda").bfloat16()
    got = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n)
    want, bound = token_definition(q, cache, table, [length], 0, dim ** -0.5)
    check(got, want, bound)


@pytest.mark.parametrize("kind", [F8, I8])
@pytest.mark.parametrize("window", [0, 400])
@pytest.mark.parametrize("spread,sharp", [(4.0, 1.0), (20.0, 1.0), (20.0, 20.0), (4.0, 200.0)])
def test_scales_and_scores_of_all_sizes(spread, sharp, window, kind):
    lengths = [700, 33, 5000]
    cache, table, n = filled(lengths, 2, 16, 64, kind, 11)
    g = torch.Generator(device="cuda").manual_seed(3)
    cache[3].mul_(torch.exp(spread * torch.randn(cache[3].shape, generator=g, device="cuda")).clamp(1e-30, 1e30))
    q = (sharp * torch.randn(3, 8, 64, generator=g, device="cuda")).bfloat16()
    got = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n, window=window)
    want, bound = token_definition(q, cache, table, lengths, window, 0.125)
    check(got, want, bound)


@pytest.mark.parametrize("kind", [F8, I8])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -100, 2.0 ** 100])
def test_scales_that_are_all_small_or_large(size, kind):
    cache, table, n = filled([300, 2000], 1, 16, 64, kind, 5)
    cache[3].copy_(torch.where(torch.isnan(cache[3]), cache[3], torch.full_like(cache[3], size)))
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    got = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n).double() / size
    want, bound = token_definition(q, (cache[0], cache[1], cache[2], cache[3] / size), table, [300, 2000], 0, 0.125)
    # (results under 2^-126 keep fewer bits than 8: as multiples of bf16's least step 2^-133)
    check(got, want, bound + (2.0 ** -133 / size if size < 1 else 0.0))


@pytest.mark.parametrize("kind", [F8, I8])
@pytest.mark.parametrize("length", [700, 9000])
@pytest.mark.parametrize("size", [lambda t: torch.where(t == 0, 0.0, -126.0), lambda t: torch.where(t == 0, 60.0, 0.0), lambda t: torch.where(t % 97 == 0, 40.0, -40.0),
                                  lambda t: t / 100.0 - 45, lambda t: 45 - t / 100.0], ids=["first", "first large", "some", "rising", "falling"])
@pytest.mark.parametrize("group", [4, 16])
def test_scores_that_rise_along_the_tokens(group, size, length, kind):
    """The running maximum moves in each step of a head whose scores rise fast, beside heads of the same group whose scores rise slowly or fall."""
    cache, table, n = filled([length], 1, 16, 64, kind, 4)
    t = torch.arange(length, device="cuda")
    page, place = table[0, t // 16].long(), t % 16
    cache[0].view(torch.uint8)[page, :, place] = torch.full((length, 1, 64), float(MOST[kind]), device="cuda").to(kind).view(torch.uint8)
    cache[2][page, :, place] = (t + 1)[:, None] / (MOST[kind] * 8)
    cache[3][page, :, place] = torch.exp2(size(t.float()))[:, None].float()
    rates = torch.tensor([0.001, 0.0, 0.3, -0.02, 0.02, 1.0, -1.0, 0.0001], device="cuda").repeat(2)[:group]
    q = (rates[None, :, None] * torch.ones(1, group, 64, device="cuda")).bfloat16()
    got = nq.nq_paged_attention(q, nq.nq_kv_pages(*cache), table, n)
    want, bound = token_definition(q, cache, table, [length], 0, 0.125)
    check(got, want, bound)
