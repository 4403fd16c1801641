"""The served decoder stack end to end: prompts, prompts behind a prefix and single tokens against the same stack in 64 bits.

Tolerance.  Rounding to e4m3 costs a value 2.6 % in the root mean square, so a product of two rounded matrices with random signs is off
by about 3.7 % of its norm, and n of them one after the other by 3.7 % * sqrt(n): two layers have eight.  An e4m3 or INT8 cache rounds keys
and values once more, as one product each does: ten.  Twice that is allowed."""
import copy
import math

import pytest
import torch

import paper_2506_17870_b200 as nq
from fp8_reference import norm
from paper_2506_17870_b200.attention import AttentionBlock, DecoderStack, main

pytestmark = pytest.mark.gpu
BF16, F8, I8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8
LIMIT = 2 * 0.037 * math.sqrt(10)


def in_64_bits(stack, x):
    """One sequence's stream [tokens, width] through the stack."""
    x, y = x.double(), None
    d = lambda t: t.detach().double()
    n = len(stack.blocks)
    for i in range(n + 1):
        b = stack.blocks[i] if i < n else None
        if y is not None:
            last = stack.blocks[i - 1]
            x = stack.how["skip_scale"] * x + stack.how["branch_scale"] * norm(y, 1, d(last.post_weight), None, 1e-6) * d(last.gate)
        h = norm(x, 1, d(b.pre_weight if b is not None else stack.final_weight), None, 1e-6)
        if b is None:
            return h
        if not isinstance(b, AttentionBlock):
            y = torch.nn.functional.gelu(h @ d(b.up).t() + d(b.up_bias)) @ d(b.down).t()
            continue
        dim, qh, kv = b.head_dim, b.q_heads, b.kv_heads
        heads = (h @ d(b.qkv).t()).view(len(x), -1, dim)
        turn = d(stack.angles)[: len(x), None]
        c, s = turn[..., : dim // 2], turn[..., dim // 2:]

        def prepared(t, w):
            t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * d(w)
            a, e = t[..., : dim // 2], t[..., dim // 2:]
            return torch.cat([a * c - e * s, e * c + a * s], -1)
        q, k = prepared(heads[:, :qh], b.q_weight), prepared(heads[:, qh:qh + kv], b.k_weight).repeat_interleave(qh // kv, 1)
        v = heads[:, qh + kv:].repeat_interleave(qh // kv, 1)
        scores = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(dim)
        scores = scores.masked_fill(torch.ones(len(x), len(x), dtype=torch.bool, device="cuda").triu(1), -math.inf)
        y = torch.einsum("hij,jhd->ihd", scores.softmax(-1), v).flatten(1) @ d(b.out).t()


def make(dim=64, kind=F8, pages=64, page_size=16, seed=1):
    torch.manual_seed(seed)
    stack = DecoderStack(2, 256, 640, 4, 2, dim, positions=512, skip_scale=0.9, branch_scale=1.1)
    with torch.no_grad():
        for b in stack.blocks:
            if isinstance(b, AttentionBlock):
                b.q_weight.add_(0.2 * torch.randn_like(b.q_weight))
                b.k_weight.add_(0.2 * torch.randn_like(b.k_weight))
    stack.freeze()
    return stack, stack.cache(pages, page_size, kind)


def near(got, want):
    assert float((got.double() - want).norm() / want.norm()) < LIMIT


@pytest.mark.parametrize("kind", [BF16, F8, I8])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_prefixes_and_tokens(dim, kind):
    stack, table = make(dim, kind)
    lengths, more = [130, 5, 64], [40, 1, 70]
    x = [torch.randn(n + m + 3, 256, device="cuda", dtype=BF16) for n, m in zip(lengths, more)]
    want = [in_64_bits(stack, v) for v in x]
    ids = [table.add() for _ in lengths]
    prompt = stack.serve(torch.cat([v[:n] for v, n in zip(x, lengths)]), table.extend(ids, lengths)).split(lengths)
    behind = stack.serve(torch.cat([v[n:n + m] for v, n, m in zip(x, lengths, more)]), table.extend(ids, more)).split(more)
    for i, (n, m) in enumerate(zip(lengths, more)):
        near(prompt[i], want[i][:n])
        near(behind[i], want[i][n:n + m])
    for t in range(3):
        out = stack.serve(torch.stack([v[-3 + t] for v in x]), table.extend(ids, [1, 1, 1]))
        for i in range(3):
            near(out[i], want[i][-3 + t])
    nq.nq_device_status()


def test_pages_of_an_ended_sequence_are_used_again_and_others_keep_theirs():
    stack, table = make(pages=12)
    x = torch.randn(3, 90, 256, device="cuda", dtype=BF16)
    a, b = table.add(), table.add()
    stack.serve(x[:2, :80].reshape(-1, 256), table.extend([a, b], [80, 80]))
    table.drop(a)
    c = table.add()
    out = stack.serve(x[2, :80], table.extend([c], [80]))
    near(out, in_64_bits(stack, x[2, :80]))
    out = stack.serve(torch.stack([x[1, 80], x[2, 80]]), table.extend([b, c], [1, 1]))
    near(out[0], in_64_bits(stack, x[1, :81])[-1])
    near(out[1], in_64_bits(stack, x[2, :81])[-1])


def test_one_token_replayed_from_a_graph():
    """A captured pass over one token of each sequence follows what the batch's tensors are set to."""
    stack, table = make(kind=F8)
    x = torch.randn(2, 60, 256, device="cuda", dtype=BF16)
    ids = [table.add(), table.add()]
    stack.serve(x[:, :50].reshape(-1, 256), table.extend(ids, [50, 50]))
    batch, stream = table.extend(ids, [1, 1]), x[:, 50].clone()
    eager = [stack.serve(stream, batch)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = stack.serve(stream, batch)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, eager[0])
    for t in range(51, 60):
        new = table.extend(ids, [1, 1])
        stream.copy_(x[:, t])
        for old, now in zip((batch.positions, batch.slots, batch.lengths, batch.table), (new.positions, new.slots, new.lengths, new.table)):
            old.copy_(now)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, stack.serve(stream, new))


def test_frozen_weights_only():
    stack, table = make()
    i = table.add()
    x = torch.randn(4, 256, device="cuda", dtype=BF16)
    batch = table.extend([i], [4])
    first = stack.serve(x, batch)
    twin = copy.deepcopy(stack.blocks[1])
    assert twin.served is not None
    twin = copy.deepcopy(stack.blocks[0])
    assert twin.served is not None and twin.pages is None and stack.blocks[0].pages is not None
    with torch.no_grad():
        stack.blocks[0].qkv.mul_(1.0)
    with pytest.raises(RuntimeError, match="freeze"):
        stack.serve(x, batch)
    stack.freeze()
    assert torch.equal(stack.serve(x, batch), first)
    with pytest.raises(RuntimeError, match="for serving"):
        stack(x)
    bare = DecoderStack(1, 256, 640, 4, 2, 64, positions=64)
    bare.freeze()
    with pytest.raises(RuntimeError, match="cache"):
        bare.serve(x, batch)


def test_the_module_runs():
    assert main() < LIMIT
