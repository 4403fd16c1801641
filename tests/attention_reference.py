"""The attention operators' definitions in 64 bits, without the library's code, and what the tests make their inputs with."""
import math

import torch

MOST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}


def quantise(x, dtype):
    """The cache's codes and scales, one fp32 rounding an operation, as the definition has them."""
    x = x.float()
    s = torch.clamp(x.abs().amax(-1) / torch.full((), MOST[dtype], device=x.device), min=2.0 ** -126)
    y = x * (torch.ones((), device=x.device) / s)[..., None]
    y = torch.clamp(y, -MOST[dtype], MOST[dtype])
    return (y.to(dtype) if dtype is torch.float8_e4m3fn else torch.round(torch.nan_to_num(y, nan=0.0)).to(dtype)), s


def empty(pages, heads, page, dim, dtype, fill=0.0, device="cuda"):
    """k, v, ks, vs of a cache full of `fill` (as values, or as scales)."""
    shape = (pages, heads, page, dim)
    if dtype is torch.bfloat16:
        return torch.full(shape, fill, dtype=dtype, device=device), torch.full(shape, fill, dtype=dtype, device=device), None, None
    ones = lambda: torch.ones(shape, dtype=torch.float32, device=device).to(dtype)
    scales = lambda: torch.full(shape[:3], fill, device=device)
    return ones(), ones(), scales(), scales()


def values(codes, scales):
    return codes.double() if scales is None else codes.double() * scales.double()[..., None]


def filled(lengths, heads, page, dim, dtype, seed=0, spare=3, hole=float("nan"), order=True):
    """(tensors of a cache, table, lengths): each sequence's tokens random, everything that belongs to none `hole`."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages, cols = sum(need) + spare, max(1, max(need, default=1))
    k, v, ks, vs = empty(pages, heads, page, dim, dtype, hole)
    perm = torch.randperm(pages, generator=g, device="cuda").int() if order else torch.arange(pages, dtype=torch.int32, device="cuda")
    table = torch.full((len(lengths), cols), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(lengths):
        table[i, : need[i]] = perm[at: at + need[i]]
        at += need[i]
        for c, s in ((k, ks), (v, vs)):
            x = torch.randn(need[i] * page, heads, dim, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(need[i] * page, heads, 1, generator=g, device="cuda"))
            x = x.view(need[i], page, heads, dim).transpose(1, 2)
            live = (torch.arange(need[i] * page, device="cuda") < n).view(need[i], 1, page).expand(need[i], heads, page)
            used = table[i, : need[i]].long()
            if s is None:
                old = c[used]
                c[used] = torch.where(live[..., None], x.to(dtype), old)
            else:
                q, sc = quantise(x, dtype)
                c.view(torch.uint8)[used] = torch.where(live[..., None], q.contiguous().view(torch.uint8), c.view(torch.uint8)[used])
                s[used] = torch.where(live, sc, s[used])
    return (k, v, ks, vs), table, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def sequence(cache, table_row, n, which):
    """Tokens 0 .. n of a sequence, [n, heads, dim] in 64 bits (pages all inside the cache)."""
    c, s = cache[which], cache[2 + which]
    page = c.shape[2]
    used = table_row[: -(-n // page)].long()
    x = values(c[used], None if s is None else s[used])
    return x.transpose(1, 2).reshape(-1, c.shape[1], c.shape[3])[:n]


def attend(q, k, v, seen, scale):
    """q [rows, heads, dim], k, v [tokens, kv_heads, dim], seen [rows, tokens] -> (y, bound): the attention in 64 bits (rows that see
    nothing: zero) and a bound of a kernel's error that counts
      weights rounded to bf16 (half a step, 2^-8 of each) and the result too;
      a score's error: a sum of dim products in fp32, each addition off by no more than a step of the running sum of magnitudes, and
      its exponential by as much (twice: in the weight and in the sum of weights)."""
    q, k, v = q.double(), k.double(), v.double()
    group = q.shape[1] // k.shape[1]
    y, bound = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    any_seen = seen.any(1)
    for h in range(q.shape[1]):
        kh, vh = k[:, h // group], v[:, h // group]
        kh = torch.where(seen.any(0)[:, None], kh, 0.0)
        vh = torch.where(seen.any(0)[:, None], vh, 0.0)
        s = (q[:, h] @ kh.t()) * scale
        s = s.masked_fill(~seen, -math.inf)
        w = torch.softmax(s, -1)
        w = torch.where(any_seen[:, None], w, 0.0)
        off = (q[:, h].abs() @ kh.abs().t()) * abs(scale)
        off = torch.where(seen, off, 0.0).amax(1, keepdim=True) * (q.shape[2] * 2.0 ** -24) * 2 + 2.0 ** -20
        y[:, h] = w @ vh
        bound[:, h] = (2.0 ** -8 + off) * (w @ vh.abs()) + 2.0 ** -8 * y[:, h].abs() + 1e-30
    return y, bound


def check(got, want, bound):
    got = got.double()
    assert bool(torch.isfinite(got).all()), "not finite"
    over = ((got - want).abs() / bound).max()
    assert float(over) <= 1.0, f"{float(over):.3g} times the bound"
