"""Caches, keys, queries and results whose offsets pass 32 bits, against the definition in 64 bits."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import attend, check, quantise, sequence
from test_gpu_prompt_attention import seen_of, starts_of

pytestmark = pytest.mark.gpu
BF16, F8, I8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8


@pytest.mark.parametrize("kind", [BF16, F8, I8])
def test_pages_past_2_to_the_32_elements(kind):
    """Tokens written to, read from and attended over the last and the first pages of a cache of 2^32 values and a few more."""
    heads, page, dim = 8, 32, 128
    pages = (1 << 32) // (heads * page * dim) + 3
    codes = lambda: torch.empty(pages, heads, page, dim, dtype=torch.uint8 if kind is not BF16 else BF16, device="cuda").view(kind)
    scales = lambda: None if kind is BF16 else torch.empty(pages, heads, page, device="cuda")
    cache = (codes(), codes(), scales(), scales())
    c = nq.nq_kv_pages(*cache)
    used = torch.tensor([pages - 1, 0, pages - 2, pages // 2 + 1], dtype=torch.int32, device="cuda")
    n = 3 * page + 5
    t = torch.arange(n, device="cuda")
    slots = (used[t // page] * page + t % page).int()
    k, v = (torch.randn(n, heads, dim, device="cuda").bfloat16() for _ in range(2))
    nq.nq_kv_cache_write(c, k, v, slots)
    for which, x in ((0, k), (1, v)):
        want = x.double() if kind is BF16 else (lambda q, s: q.double() * s.double()[..., None])(*quantise(x, kind))
        assert bool((sequence(cache, used, n, which) == want).all())
    kr, vr = nq.nq_kv_cache_read(c, used[None], torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, y_dtype=torch.float32)
    assert all(bool((got == sequence(cache, used, n, which).float()).all()) for which, got in ((0, kr), (1, vr)))        # (one rounding to fp32)
    q = torch.randn(1, 2 * heads, dim, device="cuda").bfloat16()
    y = nq.nq_paged_attention(q, c, used[None], torch.tensor([n], dtype=torch.int32, device="cuda"))
    want, bound = attend(q, sequence(cache, used, n, 0), sequence(cache, used, n, 1), torch.ones(1, n, dtype=torch.bool, device="cuda"), dim ** -0.5)
    check(y, want, bound + 2.0 ** -32 * n * float(v.abs().max()))
    # and straight from a fused projection
    x = torch.randn(n, 4 * heads * dim, device="cuda").bfloat16()
    nq.nq_qk_norm_rotate(x, None, None, q_heads=2 * heads, kv_heads=heads, cache=c, slots=slots)
    x = x.view(n, 4 * heads, dim)[:, 3 * heads:]
    assert bool((sequence(cache, used, n, 1) == (x.double() if kind is BF16 else (lambda q, s: q.double() * s.double()[..., None])(*quantise(x, kind)))).all())


@pytest.mark.parametrize("heads", [(2, 1), (1, 1)])
def test_prompts_behind_2_to_the_32_elements(heads):
    q_heads, kv_heads = heads
    dim, n, m = 64, 200, 300
    rows_q, rows_k = (1 << 32) // (q_heads * dim) + 500, (1 << 32) // (kv_heads * dim) + 500
    q, k, v, y = (torch.empty(rows, h, dim, dtype=BF16, device="cuda") for rows, h in ((rows_q, q_heads), (rows_k, kv_heads), (rows_k, kv_heads), (rows_q, q_heads)))
    at_q, at_k = rows_q - n - 7, rows_k - m - 9
    for x, at, rows in ((q, at_q, n), (k, at_k, m), (v, at_k, m)):
        x[at - 200:].fill_(float("nan"))
        x[at:at + rows].normal_()
    y[at_q - 5:] = 3.0
    nq.nq_prompt_attention(q, k, v, starts_of([n], at_q), starts_of([m], at_k), y_out=y)
    nq.nq_device_status()
    want, bound = attend(q[at_q:at_q + n], k[at_k:at_k + m], v[at_k:at_k + m], seen_of(n, m, True, 0), dim ** -0.5)
    check(y[at_q:at_q + n], want, bound)
    assert bool((y[at_q - 5:at_q] == 3).all()) and bool((y[at_q + n:] == 3).all())


def test_rotated_rows_past_2_to_the_31_elements():
    tokens, width = (1 << 31) // 512 + 9, 512
    x = torch.empty(tokens, width, dtype=BF16, device="cuda")
    x[-9:].normal_()
    x[:9].copy_(x[-9:])
    q, k = nq.nq_qk_norm_rotate(x, None, None, q_heads=4, kv_heads=2, head_dim=64)
    for y, heads in ((q, x[-9:].view(9, 8, 64)[:, :4]), (k, x[-9:].view(9, 8, 64)[:, 4:6])):
        want = heads.double() / torch.sqrt((heads.double() ** 2).mean(-1, keepdim=True) + 1e-6)
        assert torch.equal(y[-9:], y[:9])
        check(y[-9:], want, want.abs() * (2.0 ** -8 + 2.0 ** -17) + 1e-30)
