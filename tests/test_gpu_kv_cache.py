"""Head norms with rotation, the paged cache written and read back, against 64-bit definitions or bit for bit."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import empty, quantise

pytestmark = pytest.mark.gpu
BF16, F8, I8, F32 = torch.bfloat16, torch.float8_e4m3fn, torch.int8, torch.float32


def angles_of(rows, rotary):
    at = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / max(rotary, 1))
    return torch.cat([at.cos(), at.sin()], 1).float()


def definition(x, weight, angles, positions, rms, neighbours, eps):
    """Heads [tokens, heads, dim] in 64 bits, normed and turned."""
    x = x.double()
    if rms:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if weight is not None:
            x = x * weight.double()
    if angles is None:
        return x
    n = angles.shape[1]
    turn = angles.double()[positions.long()][:, None]
    c, s = turn[..., : n // 2], turn[..., n // 2:]
    y = x.clone()
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if neighbours else (x[..., : n // 2], x[..., n // 2: n])
    if neighbours:
        y[..., 0:n:2], y[..., 1:n:2] = a * c - b * s, b * c + a * s
    else:
        y[..., : n // 2], y[..., n // 2: n] = a * c - b * s, b * c + a * s
    return y


def near(got, want):
    """Half a step of the result's type; fp32 arithmetic on the way: a mean of up to 128 squares (64 steps of the rest at most), a
    root, three products and a sum, all under 2^-17 of the largest of the pair that is turned."""
    half = torch.finfo(got.dtype).eps / 2
    top = want.abs().amax(-1, keepdim=True)
    over = ((got.double() - want).abs() - half * want.abs() - 2.0 ** -17 * top).max()
    assert float(over) <= 0, float(over)


@pytest.mark.parametrize("tokens,q_heads,kv_heads,dim,rotary,neighbours,rms,weights,x_dtype,y_dtype", [
    (1, 4, 1, 128, 128, False, True, True, BF16, BF16), (3, 32, 8, 128, 128, True, True, True, BF16, BF16), (5, 5, 5, 64, 64, False, True, True, BF16, F32),
    (130, 3, 1, 64, 32, True, True, False, F32, F32), (33, 6, 2, 128, 16, False, False, False, F32, BF16), (17, 12, 12, 64, 48, False, True, True, BF16, BF16),
    (700, 8, 2, 128, 64, False, True, True, BF16, BF16), (9, 7, 1, 128, 112, True, False, False, BF16, BF16), (4001, 2, 1, 64, 0, False, True, True, BF16, BF16)])
def test_norm_and_rotation(tokens, q_heads, kv_heads, dim, rotary, neighbours, rms, weights, x_dtype, y_dtype):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    rows = (q_heads + 2 * kv_heads) * dim
    x = (3 * torch.randn(tokens, rows + 24, generator=g, device="cuda")).to(x_dtype)[:, :rows]             # a pitch of its own
    w = [1 + 0.3 * torch.randn(dim, generator=g, device="cuda") for _ in range(2)] if weights else [None, None]
    angles = angles_of(5000, rotary) if rotary else None
    positions = torch.randint(0, 5000, (tokens,), generator=g, device="cuda", dtype=torch.int32) if rotary else None
    q, k = nq.nq_qk_norm_rotate(x, angles, positions, q_heads=q_heads, kv_heads=kv_heads, norm=nq.NQ_NORM_RMS if rms else nq.NQ_NORM_NONE, q_weight=w[0],
                                k_weight=w[1], eps=1e-5, neighbours=neighbours, y_dtype=y_dtype)
    heads = x.reshape(tokens, -1, dim)
    assert q.dtype is y_dtype and k.dtype is y_dtype and q.shape == (tokens, q_heads, dim) and k.shape == (tokens, kv_heads, dim)
    near(q, definition(heads[:, :q_heads], w[0], angles, positions, rms, neighbours, 1e-5))
    near(k, definition(heads[:, q_heads:q_heads + kv_heads], w[1], angles, positions, rms, neighbours, 1e-5))


def test_rotation_of_far_positions_and_of_none():
    x = torch.randn(4, 3 * 128, device="cuda").bfloat16()
    angles = angles_of(1 << 17, 128)
    positions = torch.tensor([(1 << 17) - 1, 1 << 17, -1, 0], dtype=torch.int32, device="cuda")
    q, k = nq.nq_qk_norm_rotate(x, angles, positions, q_heads=1, kv_heads=1)
    inside = torch.tensor([0, 3], device="cuda")
    near(q[inside], definition(x.view(4, 3, 128)[inside, :1], None, angles, positions[inside], True, False, 1e-6))
    assert torch.isnan(q[1]).all() and torch.isnan(k[2]).all()
    q, _ = nq.nq_qk_norm_rotate(x, angles_of(4, 32), torch.full((4,), 9, dtype=torch.int32, device="cuda"), q_heads=1, kv_heads=1)
    assert torch.isnan(q[..., :32]).all() and torch.isfinite(q[..., 32:]).all()


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("tokens,heads,dim,page,x_dtype", [(1, 1, 64, 16, BF16), (37, 8, 128, 48, BF16), (5, 3, 64, 16, F32), (300, 5, 128, 32, F32), (3001, 2, 64, 128, BF16)])
def test_write_and_read_back(tokens, heads, dim, page, x_dtype, kind):
    g = torch.Generator(device="cuda").manual_seed(tokens + dim)
    pages = -(-tokens // page) + 2
    k, v = ((torch.randn(tokens, 2 * heads, dim, generator=g, device="cuda") * torch.exp(3 * torch.randn(tokens, 2 * heads, 1, generator=g, device="cuda")))
            .to(x_dtype)[:, i * heads:(i + 1) * heads] for i in range(2))                                   # views with a pitch of their own
    k[0, 0] = 0.0
    cache = empty(pages, heads, page, dim, kind, 7.0)
    want = [None if t is None else t.clone() for t in cache]
    perm = torch.randperm(pages * page, generator=g, device="cuda")[:tokens]
    slots = perm.int()
    if tokens > 4:
        slots[2], slots[4] = -1, pages * page                                                               # passed over
    nq.nq_kv_cache_write(nq.nq_kv_pages(*cache), k, v, slots)
    at = torch.tensor([i for i in range(tokens) if tokens <= 4 or i not in (2, 4)], device="cuda")
    where = perm[at] // page, slice(None), perm[at] % page
    for n, x in enumerate((k, v)):
        if kind is BF16:
            want[n][where] = x[at].to(BF16)
        else:
            codes, scales = quantise(x[at], kind)
            want[n].view(torch.uint8)[where] = codes.view(torch.uint8)
            want[2 + n][where] = scales
    for got, w in zip(cache, want):
        assert w is None or torch.equal(got.view(torch.uint8), w.view(torch.uint8))
    # back, through a table that names the pages in another order; rows of no sequence stay
    order = torch.randperm(pages, generator=g, device="cuda").int()
    lengths = [0, min(page + 1, (pages - 2) * page), 0, 1]
    starts = torch.tensor([3, 3, 3 + lengths[1], 3 + lengths[1], 4 + lengths[1]], dtype=torch.int32, device="cuda")
    rows = 8 + lengths[1]
    table = torch.full((4, pages + 3), -7, dtype=torch.int32, device="cuda")[:, :pages]
    table[1, :], table[3, 0] = order, order[0]
    for y_dtype in (BF16, F32):
        out = [torch.full((rows, heads, dim + 16), 3.0, dtype=y_dtype, device="cuda") for _ in range(2)]
        wide = [torch.full((rows, heads * dim + 32), 3.0, dtype=y_dtype, device="cuda") for _ in range(2)]
        views = [w[:, : heads * dim].unflatten(1, (heads, dim)) for w in wide]
        got = nq.nq_kv_cache_read(nq.nq_kv_pages(*cache), table, starts, rows, k_out=views[0], v_out=views[1])
        for n in range(2):
            c = cache[n].float() if kind is BF16 else cache[n].float() * cache[2 + n][..., None]
            c = c.to(y_dtype)[order.long()].transpose(1, 2).reshape(-1, heads, dim)
            expect = torch.full((rows, heads, dim), 3.0, dtype=y_dtype, device="cuda")
            expect[3: 3 + lengths[1]] = c[: lengths[1]]
            expect[3 + lengths[1]] = c[0]
            assert torch.equal(got[n], expect)
            assert bool((wide[n][:, heads * dim:] == 3.0).all())
        del out


def test_pages_outside_the_cache_read_as_zeros():
    cache = empty(2, 2, 16, 64, F8, 1.0)
    table = torch.tensor([[1, 2, -1, 0]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 80], dtype=torch.int32, device="cuda")                                        # 64 tokens of pages, 16 of none
    k, v = nq.nq_kv_cache_read(nq.nq_kv_pages(*cache), table, starts, 80)
    live = torch.zeros(80, dtype=torch.bool, device="cuda")
    live[:16], live[48:64] = True, True
    assert bool((k[live] == 1).all()) and bool((k[~live] == 0).all()) and bool((v[live] == 1).all()) and bool((v[~live] == 0).all())


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("tokens,q_heads,kv_heads,dim", [(1, 8, 2, 128), (3, 32, 8, 128), (70, 5, 5, 64), (2500, 4, 1, 64)])
def test_rotation_straight_to_the_cache(tokens, q_heads, kv_heads, dim, kind):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn(tokens, (q_heads + 2 * kv_heads) * dim, generator=g, device="cuda").bfloat16()
    w = 1 + 0.3 * torch.randn(dim, generator=g, device="cuda")
    angles = angles_of(999, dim)
    positions = torch.randint(0, 999, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    page, pages = 16, -(-tokens // 16) + 1
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens].int()
    cache = empty(pages, kv_heads, page, dim, kind)
    how = dict(q_heads=q_heads, kv_heads=kv_heads, q_weight=w, k_weight=w)
    q, k = nq.nq_qk_norm_rotate(x, angles, positions, cache=nq.nq_kv_pages(*cache), slots=slots, want_k=True, y_dtype=F32, **how)
    q2, k2 = nq.nq_qk_norm_rotate(x, angles, positions, y_dtype=F32, **how)
    assert torch.equal(q, q2) and torch.equal(k, k2)
    two = empty(pages, kv_heads, page, dim, kind)                                                            # the same by the two steps
    nq.nq_kv_cache_write(nq.nq_kv_pages(*two), k, x.view(tokens, -1, dim)[:, q_heads + kv_heads:].float(), slots)
    for a, b in zip(cache, two):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("kind", [F8, I8])
def test_values_that_are_no_numbers(kind):
    x = torch.randn(4, 1, 64, device="cuda")
    x[1, 0, 5], x[2, 0, 6] = float("nan"), float("-inf")
    x[3] = 0.0
    cache = empty(1, 1, 16, 64, kind, 1.0)
    slots = torch.arange(4, dtype=torch.int32, device="cuda")
    nq.nq_kv_cache_write(nq.nq_kv_pages(*cache), x, x, slots)
    s = cache[2][0, 0, :4]
    assert torch.isnan(s[1]) and s[2] == float("inf") and s[3] == 2.0 ** -126
    k, _ = nq.nq_kv_cache_read(nq.nq_kv_pages(*cache), torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                               torch.tensor([0, 4], dtype=torch.int32, device="cuda"), 4, y_dtype=F32)
    assert torch.isfinite(k[0]).all() and torch.isnan(k[1]).all() and torch.isnan(k[2]).all() and bool((k[3] == 0).all())


def test_offsets_past_32_bits():
    page, heads, dim = 128, 8, 128                                                                          # 2.1e9 bf16 elements, 4.3 GB each of k and v
    pages = (1 << 31) // (page * heads * dim) + 2
    cache = [torch.zeros(pages, heads, page, dim, dtype=BF16, device="cuda") for _ in range(2)]
    c = nq.nq_kv_pages(*cache)
    x = torch.randn(3, heads, dim, device="cuda").bfloat16()
    slots = torch.tensor([pages * page - 1, 0, (pages - 1) * page], dtype=torch.int32, device="cuda")
    nq.nq_kv_cache_write(c, x, -x, slots)
    assert torch.equal(cache[0][pages - 1, :, page - 1], x[0]) and torch.equal(cache[1][0, :, 0], -x[1]) and torch.equal(cache[0][pages - 1, :, 0], x[2])
    table = torch.tensor([[pages - 1], [0]], dtype=torch.int32, device="cuda")
    k, v = nq.nq_kv_cache_read(c, table, torch.tensor([0, page, 2 * page], dtype=torch.int32, device="cuda"), 2 * page)
    assert torch.equal(k[page - 1], x[0]) and torch.equal(k[0], x[2]) and torch.equal(v[page], -x[1])
    y = nq.nq_paged_attention(x[:2].contiguous(), c, table, torch.tensor([1, 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(y[0], -x[2]) and torch.equal(y[1], -x[1])


def test_starts_far_below_zero_have_no_pages():
    cache = empty(2, 1, 16, 64, BF16, 1.0)
    table = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([-(1 << 31), 5], dtype=torch.int32, device="cuda")
    k, v = nq.nq_kv_cache_read(nq.nq_kv_pages(*cache), table, starts, 5)
    assert bool((k == 0).all()) and bool((v == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_queries_in_place(dtype):
    import ctypes
    x = torch.randn(600, (8 + 2 * 2) * 128, device="cuda").to(dtype)
    angles = angles_of(700, 128)
    positions = torch.arange(600, dtype=torch.int32, device="cuda")
    want, _ = nq.nq_qk_norm_rotate(x, angles, positions, q_heads=8, kv_heads=2, y_dtype=dtype)
    before = x.clone()
    code = nq.NQ_BF16 if dtype is BF16 else nq.NQ_F32
    k = torch.empty(600, 256, dtype=dtype, device="cuda")
    d = nq.nq_qk_desc(600, 1536, 1536, 256, 700, code, code, 8, 2, 128, 128, nq.NQ_NORM_RMS, 0, 1e-6)
    assert nq.lib().nq_qk_norm_rotate(ctypes.addressof(d), x.data_ptr(), None, None, angles.data_ptr(), positions.data_ptr(), x.data_ptr(), k.data_ptr(),
                                      None, None, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(x[:, :1024].view(600, 8, 128), want) and torch.equal(x[:, 1024:], before[:, 1024:])
