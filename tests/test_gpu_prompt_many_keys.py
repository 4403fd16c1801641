"""Attention of prompts over so many keys that a row's sums have to be kept in parts, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import attend, check
from test_gpu_prompt_attention import inputs, seen_of, starts_of

pytestmark = pytest.mark.gpu


def one_query_a_head(q, k, v, scale):
    """The definition for rows that see all keys, a head at a time and the keys in pieces (64 bits take room)."""
    y = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    group = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        s = torch.cat([q[:, h].double() @ part.double().t() for part in k[:, h // group].split(1 << 18)], 1) * scale
        w = torch.softmax(s, -1)
        y[:, h] = sum(a @ b.double() for a, b in zip(w.split(1 << 18, 1), v[:, h // group].split(1 << 18)))
    return y


@pytest.mark.parametrize("dim,heads,keys", [(64, (2, 1), 1 << 22), (64, (3, 3), 1 << 20), (128, (1, 1), (1 << 22) + 77), (128, (4, 2), 1 << 20)])
@pytest.mark.parametrize("size", [0.0, 1.0])
def test_values_of_one_sign_lose_nothing_to_their_number(size, dim, heads, keys):
    """Weights and result are rounded to bf16, half a step of 2^-8 each, which is 2^-8 of the result, for the weights' roundings have both signs: their
    mean over 2^10 keys that hold the weight would be off by 2^-8 2^-5 three times as often as not.  Beside that, sums of n products in parts of
    2^16: n 2^-27 of the part at most, 2^-11, and the parts' own additions, 2^-24 each."""
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, _ = inputs(3, keys, *heads, dim)
    q = (size * q.float()).bfloat16()
    v = (0.5 + torch.rand(keys, heads[1], dim, generator=g, device="cuda")).bfloat16()
    y = nq.nq_prompt_attention(q, k, v, starts_of([3]), starts_of([keys]), causal=False)
    nq.nq_device_status()
    want = one_query_a_head(q, k, v, dim ** -0.5)
    off = ((y.double() - want) / want)
    assert float(off.abs().max()) <= 2 ** -8 + 2 ** -11
    assert abs(float(off.mean())) <= 2 ** -10                               # no lean to one side


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [(2, 1), (1, 1)])
@pytest.mark.parametrize("keys", [65536 - 40, 65536, 65537, 65536 + 64, 65536 + 65, 131072 + 1, 140000])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 70000), (False, 0)])
def test_where_the_parts_meet(causal, window, keys, heads, dim):
    rows = 150
    q, k, v = inputs(rows + 20, keys + 20, *heads, dim, keys)
    y = nq.nq_prompt_attention(q, k, v, starts_of([rows, 20]), starts_of([keys, 20]), causal=causal, window=window)
    nq.nq_device_status()
    for a, b, n, m in ((0, 0, rows, keys), (rows, keys, 20, 20)):
        want, bound = attend(q[a:a + n], k[b:b + m], v[b:b + m], seen_of(n, m, causal, window), dim ** -0.5)
        check(y[a:a + n], want, bound)
    assert torch.equal(y, nq.nq_prompt_attention(q, k, v, starts_of([rows, 20]), starts_of([keys, 20]), causal=causal, window=window))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("slope", [1.0, -1.0, 0.0])
def test_maxima_that_move_between_the_parts(slope, dim):
    """Scores that rise or fall by some hundreds along the keys, and a row whose first part sees nothing but minus infinity."""
    keys = 150000
    q, k, v = inputs(2, keys, 1, 1, dim)
    k = (0.1 * k.float() + (slope * torch.arange(keys, device="cuda") / keys * 400 / dim ** 0.5)[:, None, None]).bfloat16()
    q = torch.ones_like(q)
    if slope == 0.0:
        k[:70000, :, 0] = -math.inf
    y = nq.nq_prompt_attention(q, k, v, starts_of([2]), starts_of([keys]), causal=False)
    at = slice(70000, None) if slope == 0.0 else slice(None)
    want, bound = attend(q, k[at], v[at], torch.ones(2, len(k[at]), dtype=torch.bool, device="cuda"), dim ** -0.5)
    check(y, want, bound)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("keys", [65536 + 40, 65536 + 64, 131072 + 33])
def test_no_numbers_hidden_in_the_first_step_of_a_part(keys, bad, dim):
    """The step that starts a part is the one that hides keys, so its product is made by hand."""
    rows = 30
    q, k, v = inputs(rows, keys, 2, 1, dim)
    clean = v.clone()
    v[keys - 5] = bad
    clean[keys - 5] = 0.0
    y = nq.nq_prompt_attention(q, k, v, starts_of([rows]), starts_of([keys]))
    nq.nq_device_status()
    want, bound = attend(q, k, clean, seen_of(rows, keys, True, 0), dim ** -0.5)
    check(y[:rows - 5], want[:rows - 5], bound[:rows - 5])
    assert not torch.isfinite(y[rows - 5:]).all(-1).any()
