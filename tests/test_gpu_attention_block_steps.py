"""Each step of a served attention block against its definition in 64 bits, on the operands that the step before it left: positions, pages and
sequences are the test's own."""
import pytest
import torch

from attention_reference import attend, check, sequence
from paper_2506_17870_b200 import binding
from paper_2506_17870_b200.attention import AttentionBlock
from test_gpu_attention_block import make

pytestmark = pytest.mark.gpu
BF16, F8, I8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8


@pytest.fixture
def calls(monkeypatch):
    made = []

    def recorded(name):
        call = getattr(binding, name)

        def wrapper(*args, **kwargs):
            out = call(*args, **kwargs)
            made.append((name, args, kwargs, out))
            return out
        monkeypatch.setattr(binding, name, wrapper)
    for name in ("nq_fp8_gemm", "nq_fp8_quantize", "nq_qk_norm_rotate", "nq_kv_cache_read", "nq_paged_attention", "nq_prompt_attention", "nq_block_norm"):
        recorded(name)
    return made


def turned(x, weight, positions):
    """Heads [tokens, heads, dim] normed and turned, and a bound without the rounding to the output's type: sums of dim squares in fp32, 2^-24
    each of the sum, and a few operations more."""
    dim = x.shape[-1]
    x = x.double()
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.double()
    at = positions.double()[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    c, s = at.cos()[:, None], at.sin()[:, None]
    a, b = x[..., : dim // 2], x[..., dim // 2:]
    size = (a.abs() + b.abs()) * (dim + 8) * 2.0 ** -24
    return torch.cat([a * c - b * s, b * c + a * s], -1), torch.cat([size, size], -1)


def stored(x, kind, scales):
    """How far a stored value may be from x: half a step of its type."""
    if kind is BF16:
        return 2.0 ** -8 * x.abs()
    s = scales.double()[..., None]
    return 2.0 ** -4 * x.abs() + 2.0 ** -10 * s if kind is F8 else 0.5 * s + 2.0 ** -16 * x.abs()


def one_pass(stack, calls, x, table, ids, before, counts, kind):
    """Serves counts[i] new tokens of sequences that have before[i], and checks each attention block."""
    calls.clear()
    batch = table.extend(ids, counts)
    stack.serve(x, batch)
    blocks = [b for b in stack.blocks if isinstance(b, AttentionBlock)]
    rotations = [i for i, c in enumerate(calls) if c[0] == "nq_qk_norm_rotate"]
    assert len(rotations) == len(blocks)
    positions = torch.cat([torch.arange(n, n + c, device="cuda") for n, c in zip(before, counts)])
    for b, at in zip(blocks, rotations):
        qh, kv, dim = b.q_heads, b.kv_heads, b.head_dim
        name, args, _, out = calls[at - 1]                                            # the fused projection, of what the norm left
        norm = calls[at - 2]
        assert name == "nq_fp8_gemm" and norm[0] == "nq_block_norm" and args[0] is norm[3][1] and args[1] is norm[3][2]
        assert args[2] is b.served[0].q and args[3] is b.served[0].s
        heads = out.view(sum(counts), -1, dim)
        q, k = calls[at][3]
        assert calls[at][1][0] is out
        want, off = turned(heads[:, :qh], b.q_weight, positions)
        check(q, want, off + 2.0 ** -8 * want.abs() + 1e-30)
        k64, k_off = turned(heads[:, qh:qh + kv], b.k_weight, positions)
        v64 = heads[:, qh + kv:].double()
        cache = b.pages.tensors
        a = 0
        for i, (n, c) in enumerate(zip(before, counts)):                             # what the cache has of the new tokens
            if c == 0:
                continue
            for which, x64, more in ((0, k64, k_off), (1, v64, torch.zeros_like(v64))):
                got = sequence(cache, batch.table[i], n + c, which)[n:]
                scales = None if kind is BF16 else sequence((cache[2][..., None], cache[3][..., None], None, None), batch.table[i], n + c, which)[n:, :, 0]
                check(got, x64[a:a + c], stored(x64[a:a + c], kind, scales) + 2 * more[a:a + c] + 1e-30)
            a += c
        later = calls[at + 1:]
        if any(before) and any(c != 1 for c in counts):                              # behind a prefix: the cache's values, rounded to bf16
            name, _, _, (kr, vr) = later.pop(0)
            assert name == "nq_kv_cache_read"
            for which, got in ((0, kr), (1, vr)):
                assert torch.equal(got, torch.cat([sequence(cache, batch.table[i], n + c, which) for i, (n, c) in enumerate(zip(before, counts))]).float().bfloat16())
        name, args, _, y = later[0]
        single = all(c == 1 for c in counts)
        assert name == ("nq_paged_attention" if single else "nq_prompt_attention") and args[0] is q
        a = first = 0
        for i, (n, c) in enumerate(zip(before, counts)):
            if single:
                keys, values = sequence(cache, batch.table[i], n + 1, 0), sequence(cache, batch.table[i], n + 1, 1)
            elif any(before):
                keys, values = kr[first:first + n + c], vr[first:first + n + c]
            else:
                keys, values = k[a:a + c], heads[a:a + c, qh + kv:]
            seen = torch.arange(n + c, device="cuda")[None] <= torch.arange(n, n + c, device="cuda")[:, None]
            if c == 0:
                first += n
                continue
            want, bound = attend(q[a:a + c], keys, values, seen, dim ** -0.5)
            # (8-bit values: weights under 2^-32 of the largest are lost, as many as there are tokens)
            check(y[a:a + c], want, bound + (0.0 if kind is BF16 else 2.0 ** -32 * (n + c) * float(values.abs().max())))
            a, first = a + c, first + n + c
        assert later[1][0] == "nq_fp8_quantize" and torch.equal(later[1][1][0], y.flatten(1))
        name, args, _, out = later[2]
        assert name == "nq_fp8_gemm" and args[0] is later[1][3][0] and args[1] is later[1][3][1] and args[2] is b.served[1].q and args[3] is b.served[1].s
        assert later[3][0] == "nq_block_norm" and any(t is out for t in later[3][1])


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_prefixes_and_tokens(dim, kind, calls):
    stack, table = make(dim, kind)
    before, ids = [0, 0, 0], [table.add() for _ in range(3)]
    for counts in ([130, 5, 64], [40, 1, 70], [1, 1, 1], [1, 0, 3], [1, 1, 1]):
        one_pass(stack, calls, torch.randn(sum(counts), 256, device="cuda", dtype=BF16), table, ids, before, counts, kind)
        before = [n + c for n, c in zip(before, counts)]
    table.drop(ids[1])
    ids[1], before[1] = table.add(), 0                                               # a new sequence beside two that go on, in pages that another had
    one_pass(stack, calls, torch.randn(22, 256, device="cuda", dtype=BF16), table, ids, before, [1, 20, 1], kind)


def test_no_new_tokens_at_all():
    stack, table = make()
    a = table.add()
    x = torch.randn(3, 256, device="cuda", dtype=BF16)
    assert stack.serve(x[:0], table.extend([a], [0])).shape == (0, 256)
    stack.serve(x, table.extend([a], [3]))
    assert stack.serve(x[:0], table.extend([a], [0])).shape == (0, 256) and stack.serve(x[:0], table.extend([], [])).shape == (0, 256)
