"""Cases of the attention operators of a served transformer: the norm of queries and keys for each head with the position
rotation, the paged key-value cache as it is written (and quantised) and read back, the attention of one new token over that
cache, and the attention over whole prompts of different lengths packed behind one another.

Layouts.  The cache is k and v [pages, kv_heads, page_size, head_dim] in bf16, e4m3 or INT8, the latter two with an fp32 scale
for each token and head, ks and vs [pages, kv_heads, page_size]; a token's slot is page * page_size + its place in the page.
`table` [sequences, pages] lists each sequence's pages, `starts` [sequences + 1] where each packed sequence begins.
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
_SIZE = {"bf16": 2, "f32": 4, "fp8": 1, "int8": 1}
_MOST = {"fp8": 448.0, "int8": 127.0}
_EPS = 1e-6


# ----------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # three sequences get a token each: their fused projection, normed, rotated, keys and values put into the cache; all latency
        dict(name="rotate 3 tokens to cache", op="rotate", tokens=3, q_heads=32, kv_heads=8, dim=128, rotary=128, pairs="halves", x="bf16", cache="fp8", page=16),
        # the same for a long batch of prompts, keys left dense for the attention over the prompt
        dict(name="rotate prompts", op="rotate", tokens=16384, q_heads=32, kv_heads=8, dim=128, rotary=128, pairs="halves", x="bf16", cache="none", page=0),
        # a token each for 37 sequences, an odd number, into an e4m3 cache
        dict(name="write 37 tokens", op="write", tokens=37, kv_heads=8, dim=128, x="bf16", cache="fp8", page=16),
        # prompts of 20011 tokens with twelve heads of 64, as the repository's image transformer has
        dict(name="write prompts", op="write", tokens=20011, kv_heads=12, dim=64, x="bf16", cache="fp8", page=64),
        # one prefix of odd length comes back from an INT8 cache ahead of a longer prompt
        dict(name="read 1 prefix", op="read", seqs=1, longest=701, kv_heads=8, dim=128, cache="int8", page=16, x="bf16"),
        # the prefixes of 16 sequences of different lengths
        dict(name="read 16 prefixes", op="read", seqs=16, longest=8192, kv_heads=8, dim=128, cache="fp8", page=32, x="bf16"),
        # one conversation, one new token: latency
        dict(name="token of 1 sequence", op="token", seqs=1, longest=1501, q_heads=32, kv_heads=8, dim=128, cache="int8", page=16, window=0),
        # one very long context: the work has to be split over its length
        dict(name="token of 1 long sequence", op="token", seqs=1, longest=131072, q_heads=32, kv_heads=8, dim=128, cache="fp8", page=64, window=0),
        # a full batch of conversations of different lengths
        dict(name="token of 64 sequences", op="token", seqs=64, longest=8192, q_heads=32, kv_heads=8, dim=128, cache="bf16", page=16, window=0),
        # the repository's image transformer: 64 images of 197 tokens, every token sees its whole image
        dict(name="prompt 64 images", op="prompt", seqs=64, longest=197, spread="equal", prefix=0, q_heads=12, kv_heads=12, dim=64, causal=False, window=0),
        # five prompts of different odd lengths, packed
        dict(name="prompt 5 packed", op="prompt", seqs=5, longest=2903, spread="ragged", prefix=0, q_heads=32, kv_heads=8, dim=128, causal=True, window=0),
        # one long prompt: all matrix work
        dict(name="prompt 1 long", op="prompt", seqs=1, longest=16384, spread="equal", prefix=0, q_heads=8, kv_heads=2, dim=128, causal=True, window=0),
    ]


def _size(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rotate", "write", "read", "token", "token", "prompt", "prompt"])
    dim, kv_heads, page = rng.choice([64, 128]), rng.choice([1, 2, 4, 5, 8, 12]), rng.choice([16, 32, 48, 64, 128])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
    cache = rng.choice(["bf16", "fp8", "int8"])
    if op in ("rotate", "write"):
        tokens = _size(rng, 1, 16384)
        x = rng.choice(["bf16", "bf16", "f32"])
        if op == "write":
            return dict(op=op, tokens=tokens, kv_heads=kv_heads, dim=dim, x=x, cache=cache, page=page)
        while tokens * (group + 2) * kv_heads * dim * _SIZE[x] > 16384 * 48 * 128 * 2:
            tokens = -(-tokens // 2)
        return dict(op=op, tokens=tokens, q_heads=group * kv_heads, kv_heads=kv_heads, dim=dim, rotary=rng.choice([dim, dim, dim // 2, 16]),
                    pairs=rng.choice(["halves", "neighbours"]), x=x, cache=rng.choice([cache, "none"]), page=page)
    if op in ("read", "token"):
        seqs, longest = _size(rng, 1, 256), _size(rng, 1, 131072)
        while seqs * longest * kv_heads * dim * _SIZE[cache] > 64 * 8192 * 8 * 128 * (1 if op == "read" else 2):
            if seqs > 1 and rng.random() < 0.5:
                seqs = -(-seqs // 2)
            else:
                longest = -(-longest // 2)
        if op == "read":
            while seqs * longest * kv_heads * dim > 16 * 8192 * 8 * 128:
                longest = -(-longest // 2)
            return dict(op=op, seqs=seqs, longest=longest, kv_heads=kv_heads, dim=dim, cache=cache, page=page, x=rng.choice(["bf16", "bf16", "f32"]))
        while seqs * longest * kv_heads * (dim + 2 * group) > 64 * 8192 * 8 * 160:
            longest = -(-longest // 2)
        return dict(op=op, seqs=seqs, longest=longest, q_heads=group * kv_heads, kv_heads=kv_heads, dim=dim, cache=cache, page=page,
                    window=_size(rng, 1, max(2, longest)) if rng.random() < 0.3 else 0)
    seqs, longest = _size(rng, 1, 64), _size(rng, 1, 16384)
    prefix = _size(rng, 1, 4096) if rng.random() < 0.3 else 0
    while seqs * longest * (longest + prefix) * group * kv_heads > 16384 * 16384 * 6:
        if seqs > 1 and rng.random() < 0.5:
            seqs = -(-seqs // 2)
        else:
            longest, prefix = -(-longest // 2), prefix // 2
    return dict(op=op, seqs=seqs, longest=longest, spread=rng.choice(["equal", "ragged", "ragged"]), prefix=prefix, q_heads=group * kv_heads,
                kv_heads=kv_heads, dim=dim, causal=rng.random() < 0.8, window=_size(rng, 1, max(2, longest)) if rng.random() < 0.25 else 0)


def _lengths(case):
    """The sequences' lengths: one of them the longest, the others anything from one token on (from a sixteenth of it for a
    cache, whose sequences have a prompt behind them)."""
    n, longest = case["seqs"], case["longest"]
    if case.get("spread") == "equal":
        return [longest] * n
    r = random.Random(1000003 * n + longest)
    low = max(1, longest // 16) if case["op"] != "prompt" else 1
    got = [r.randint(low, longest) for _ in range(n)]
    got[r.randrange(n)] = longest
    return got


# ---------------------------------------------------------------------------------------------------------- the inputs
class _Make:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def heads(self, tokens, heads, dim):
        """Normal values whose channels differ in size, some of them much larger, as keys have them."""
        c = torch.exp(0.4 * self.normal(heads, dim))
        return self.normal(tokens, heads, dim) * torch.where(torch.rand(heads, dim, generator=self.g, device="cuda") < 0.01, 6.0 * c, c)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _empty_cache(pages, case):
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    kind = case["cache"]
    codes = lambda: torch.zeros(shape, dtype=torch.bfloat16, device="cuda") if kind == "bf16" else torch.zeros(
        shape, dtype=torch.uint8, device="cuda").view(_TYPES[kind])
    scales = lambda: None if kind == "bf16" else torch.zeros(shape[:3], device="cuda")
    return dict(k=codes(), v=codes(), ks=scales(), vs=scales())


def _angles(rows, rotary):
    """cos and sin of position / 10000^(2 i / rotary), [positions, rotary]: the cosines, then the sines."""
    at = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (
        -torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    return torch.cat([at.cos(), at.sin()], 1).float()


def prepare(case, seed):
    make = _Make(seed)
    op, st = case["op"], dict(case=case)
    if op in ("rotate", "write"):
        tokens, kv, dim, kind = case["tokens"], case["kv_heads"], case["dim"], _TYPES[case["x"]]
        if op == "rotate":
            st["x"] = make.heads(tokens, case["q_heads"] + 2 * kv, dim).to(kind).view(tokens, -1)
            st["q_weight"], st["k_weight"] = 1.0 + 0.2 * make.normal(dim), 1.0 + 0.2 * make.normal(dim)
            st["positions"] = torch.randint(0, 32768, (tokens,), generator=make.g, device="cuda", dtype=torch.int32)
            st["angles"] = _angles(32768, case["rotary"])
        else:
            st["k"], st["v"] = make.heads(tokens, kv, dim).to(kind), make.heads(tokens, kv, dim).to(kind)
        if case["cache"] != "none":
            pages = -(-tokens // case["page"]) + 2
            st["cache"] = _empty_cache(pages, case)
            st["slots"] = make.order(pages * case["page"])[:tokens].int()
        return st
    lengths = _lengths(case)
    st["lengths_host"] = lengths
    if op in ("read", "token"):
        page, kv, dim = case["page"], case["kv_heads"], case["dim"]
        most = -(-case["longest"] // page)
        pages = sum(-(-n // page) for n in lengths) + 1
        st["cache"] = _empty_cache(pages, case)
        for name in ("k", "v"):
            x = make.heads(pages * page, kv, dim).view(pages, page, kv, dim).transpose(1, 2).contiguous()
            if case["cache"] == "bf16":
                st["cache"][name] = x.bfloat16()
            else:
                st["cache"][name], st["cache"][name + "s"] = _quantise(x, case["cache"])
        order, at, table = make.order(pages).int(), 0, torch.zeros(len(lengths), most, dtype=torch.int32, device="cuda")
        for i, n in enumerate(lengths):
            need = -(-n // page)
            table[i, :need] = order[at:at + need]
            at += need
        st["table"], st["lengths"] = table, _int(lengths)
        if op == "read":
            st["starts"] = _int(_starts(lengths))
        else:
            st["q"] = (make.normal(len(lengths), case["q_heads"], dim)).bfloat16()
        return st
    st["starts_q"] = _int(_starts(lengths))
    st["starts_k"] = _int(_starts([n + case["prefix"] for n in lengths]))
    total, dim = sum(lengths), case["dim"]
    total_k = total + len(lengths) * case["prefix"]
    st["q"] = make.normal(total, case["q_heads"], dim).bfloat16()
    st["k"], st["v"] = make.heads(total_k, case["kv_heads"], dim).bfloat16(), make.heads(total_k, case["kv_heads"], dim).bfloat16()
    return st


# ------------------------------------------------------------------------------------------------------- the operators
def _cache_out(c, kind):
    """The cache as values: bf16 and e4m3 as they are, INT8 as what it stands for."""
    if kind == "bf16":
        return c["k"], c["v"]
    if kind == "fp8":
        return c["k"], c["v"], c["ks"], c["vs"]
    return tuple((c[n].float() * c[n + "s"][..., None]).bfloat16() for n in ("k", "v"))


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"rotate": _plain_rotate, "write": _plain_write, "read": _plain_read, "token": _plain_token, "prompt": _plain_prompt}[op](st)
    import paper_2506_17870_b200 as nq
    cache = None
    if "cache" in st:
        cache = nq.nq_kv_pages(**st["cache"])
    if op == "rotate":
        q, k = nq.nq_qk_norm_rotate(st["x"], st["angles"], st["positions"], q_heads=case["q_heads"], kv_heads=case["kv_heads"],
                                    norm=nq.NQ_NORM_RMS, q_weight=st["q_weight"], k_weight=st["k_weight"], eps=_EPS,
                                    neighbours=case["pairs"] == "neighbours", cache=cache, slots=st.get("slots"))
        return (q, k) if cache is None else (q,) + _cache_out(st["cache"], case["cache"])
    if op == "write":
        nq.nq_kv_cache_write(cache, st["k"], st["v"], st["slots"])
        return _cache_out(st["cache"], case["cache"])
    if op == "read":
        return nq.nq_kv_cache_read(cache, st["table"], st["starts"], sum(st["lengths_host"]), y_dtype=_TYPES[case["x"]])
    if op == "token":
        return nq.nq_paged_attention(st["q"], cache, st["table"], st["lengths"], window=case["window"])
    return nq.nq_prompt_attention(st["q"], st["k"], st["v"], st["starts_q"], st["starts_k"], causal=case["causal"], window=case["window"])


# -------------------------------------------------------------------------------------------------------- plain forms
def _quantise(x, kind):
    """x [..., dim] in 32 bits -> its codes, and a scale for each row."""
    s = torch.clamp(x.abs().amax(-1) / torch.full((), _MOST[kind], device=x.device), min=2.0 ** -126)
    y = torch.clamp(x * (1.0 / s)[..., None], -_MOST[kind], _MOST[kind])
    return (y.to(torch.float8_e4m3fn) if kind == "fp8" else torch.round(y).to(torch.int8)), s


def _plain_store(cache, kind, slots, k, v):
    """Tokens of k, v [tokens, kv_heads, dim] in 32 bits into their slots."""
    page = cache["k"].shape[2]
    at, within = slots.long() // page, slots.long() % page
    if kind == "bf16":
        cache["k"][at, :, within] = k.bfloat16()
        cache["v"][at, :, within] = v.bfloat16()
        return
    qk, sk = _quantise(k, kind)
    qv, sv = _quantise(v, kind)
    cache["k"].view(torch.uint8)[at, :, within] = qk.view(torch.uint8)
    cache["v"].view(torch.uint8)[at, :, within] = qv.view(torch.uint8)
    cache["ks"][at, :, within] = sk
    cache["vs"][at, :, within] = sv


def _plain_turn(x, angles, pairs):
    """Rotates the first values of each head [tokens, heads, dim] by the angles [tokens, rotary]."""
    rotary = angles.shape[1]
    c, s = angles[:, None, : rotary // 2], angles[:, None, rotary // 2:]
    if pairs == "halves":
        a, b = x[..., : rotary // 2], x[..., rotary // 2: rotary]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:rotary:2], x[..., 1:rotary:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned, x[..., rotary:]], -1)


def _plain_rotate(st):
    case = st["case"]
    qh, kv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    x = st["x"].view(-1, qh + 2 * kv, dim).float()
    angles = st["angles"][st["positions"].long()]
    normed = lambda t, w: t * torch.rsqrt((t * t).mean(-1, keepdim=True) + _EPS) * w
    q = _plain_turn(normed(x[:, :qh], st["q_weight"]), angles, case["pairs"]).bfloat16()
    k = _plain_turn(normed(x[:, qh:qh + kv], st["k_weight"]), angles, case["pairs"])
    if case["cache"] == "none":
        return q, k.bfloat16()
    _plain_store(st["cache"], case["cache"], st["slots"], k, x[:, qh + kv:])
    return (q,) + _cache_out(st["cache"], case["cache"])


def _plain_write(st):
    kind = st["case"]["cache"]
    _plain_store(st["cache"], kind, st["slots"], st["k"].float(), st["v"].float())
    return _cache_out(st["cache"], kind)


def _plain_gather(st, name, tokens_at):
    """Rows of the cache in 32 bits: [tokens, kv_heads, dim] for (page, place) pairs."""
    c = st["cache"]
    x = c[name][tokens_at[0], :, tokens_at[1]].float()
    return x if c[name + "s"] is None else x * c[name + "s"][tokens_at[0], :, tokens_at[1]][..., None]


def _plain_read(st):
    page, starts = st["case"]["page"], st["starts"].long()
    row = torch.arange(sum(st["lengths_host"]), device="cuda")
    seq = torch.searchsorted(starts, row, right=True) - 1
    t = row - starts[seq]
    at = st["table"].long()[seq, t // page], t % page
    kind = _TYPES[st["case"]["x"]]
    return _plain_gather(st, "k", at).to(kind), _plain_gather(st, "v", at).to(kind)


def _plain_softmax(s, seen):
    """Softmax of s over its last dimension where `seen`; zero where nothing is."""
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, 1.0)


def _plain_token(st):
    case = st["case"]
    n, longest, kv, dim, page = case["seqs"], case["longest"], case["kv_heads"], case["dim"], case["page"]
    t = torch.arange(longest, device="cuda")
    at = st["table"].long()[:, t // page], (t % page).expand(n, longest)
    length = st["lengths"].long()[:, None]
    seen = t < length
    if case["window"]:
        seen = seen & (t >= length - case["window"])
    k = _plain_gather(st, "k", at)                                        # [sequences, tokens, kv_heads, dim]
    s = torch.einsum("nhgd,nthd->nhgt", st["q"].float().view(n, kv, -1, dim), k) * dim ** -0.5
    del k
    p = _plain_softmax(s, seen[:, None, None])
    v = _plain_gather(st, "v", at)
    v = torch.where(seen[:, :, None, None], v, 0.0)
    return torch.einsum("nhgt,nthd->nhgd", p, v).reshape(n, -1, dim).bfloat16()


def _plain_prompt(st):
    case = st["case"]
    n, kv, group, dim = case["seqs"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    rows, cols = case["longest"], case["longest"] + case["prefix"]
    i, j = torch.arange(rows, device="cuda"), torch.arange(cols, device="cuda")
    sq, sk = st["starts_q"].long(), st["starts_k"].long()
    lq, lk = (sq[1:] - sq[:-1])[:, None, None], (sk[1:] - sk[:-1])[:, None, None]
    seen = (i[:, None] < lq) & (j[None, :] < lk)
    if case["causal"]:
        seen = seen & (j[None, :] <= i[:, None] + (lk - lq))
    if case["window"]:
        seen = seen & (j[None, :] > i[:, None] + (lk - lq) - case["window"])
    padded = lambda x, s, m: x[(s[:-1, None] + m).clamp(max=len(x) - 1)].float()           # [sequences, tokens, heads, dim]
    q = padded(st["q"], sq, i).view(n, rows, kv, group, dim).permute(0, 2, 3, 1, 4).reshape(n, kv, group * rows, dim)
    k, v = (padded(st[name], sk, j).transpose(1, 2) for name in ("k", "v"))
    s = (torch.matmul(q, k.transpose(-1, -2)) * dim ** -0.5).view(n, kv, group, rows, cols)
    p = _plain_softmax(s, seen[:, None, None])
    del s
    o = torch.matmul(p.view(n, kv, group * rows, cols), v).view(n, kv, group, rows, dim)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, rows, kv * group, dim)
    return o[(i < lq[:, 0])].bfloat16()


# --------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_scale(x, kind):
    return x.abs().max(dim=-1).values / _MOST[kind]


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; in the place of e4m3 codes, the values that are rounded to them."""
    st = prepare(case, seed)
    op, dim, kv = case["op"], case["dim"], case["kv_heads"]
    if op in ("rotate", "write"):
        if op == "rotate":
            qh, half = case["q_heads"], case["rotary"] // 2
            x = st["x"].double().view(case["tokens"], -1, dim)
            turn = st["angles"].double()[st["positions"].long()]
            turn = torch.complex(turn[:, :half], turn[:, half:])[:, None]

            def normed(t, w):
                t = t / torch.sqrt((t ** 2).sum(-1, keepdim=True) / dim + _EPS) * w.double()
                if case["pairs"] == "halves":
                    z = torch.complex(t[..., :half], t[..., half:2 * half]) * turn
                    t[..., :half], t[..., half:2 * half] = z.real, z.imag
                else:
                    z = torch.view_as_complex(t[..., :2 * half].reshape(*t.shape[:2], half, 2).contiguous()) * turn
                    t[..., :2 * half] = torch.view_as_real(z).reshape(*t.shape[:2], 2 * half)
                return t
            q, k, v = normed(x[:, :qh], st["q_weight"]), normed(x[:, qh:qh + kv], st["k_weight"]), x[:, qh + kv:]
            if case["cache"] == "none":
                return q, k
        else:
            q, k, v = None, st["k"].double(), st["v"].double()
        kind, slots, out = case["cache"], st["slots"].long(), []
        scales = []
        for t in (k, v):
            s = torch.ones(t.shape[:2], dtype=torch.float64, device="cuda") if kind == "bf16" else _exact_scale(t, kind)
            where = slots // case["page"], slice(None), slots % case["page"]
            values = torch.zeros(st["cache"]["k"].shape, dtype=torch.float64, device="cuda")
            values[where] = t / s[..., None] if kind == "fp8" else t
            out.append(values)
            held = torch.zeros(values.shape[:3], dtype=torch.float64, device="cuda")
            held[where] = s
            scales.append(held)
        if kind == "fp8":
            out += scales
        return tuple(out) if q is None else (q, *out)
    lengths = st["lengths_host"]
    if op in ("read", "token"):
        page, c = case["page"], st["cache"]

        def sequence(i, name):
            used = st["table"][i, : -(-lengths[i] // page)].long()
            x = c[name][used].double()
            if c[name + "s"] is not None:
                x = x * c[name + "s"][used].double().unsqueeze(-1)
            return x.transpose(1, 2).reshape(-1, kv, dim)[: lengths[i]]
        if op == "read":
            return tuple(torch.cat([sequence(i, name) for i in range(len(lengths))]) for name in ("k", "v"))
        out = []
        for i, n in enumerate(lengths):
            first = max(0, n - case["window"]) if case["window"] else 0
            k, v = sequence(i, "k")[first:], sequence(i, "v")[first:]
            q = st["q"][i].double().view(kv, -1, dim)
            w = torch.softmax(torch.matmul(q, k.permute(1, 2, 0)) / math.sqrt(dim), -1)
            out.append(torch.matmul(w, v.transpose(0, 1)).reshape(-1, dim))
        return torch.stack(out)
    sq, sk, group = _starts(lengths), _starts([n + case["prefix"] for n in lengths]), case["q_heads"] // kv
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for i, n in enumerate(lengths):
        m = n + case["prefix"]
        for h in range(kv):
            k, v = st["k"][sk[i]:sk[i + 1], h].double(), st["v"][sk[i]:sk[i + 1], h].double()
            for a in range(0, n, 2048):
                b = min(n, a + 2048)
                hidden = torch.zeros(b - a, m, dtype=torch.bool, device="cuda")
                gap = torch.arange(m, device="cuda")[None, :] - (torch.arange(a, b, device="cuda")[:, None] + m - n)
                if case["causal"]:
                    hidden |= gap > 0
                if case["window"]:
                    hidden |= gap <= -case["window"]
                q = st["q"][sq[i] + a:sq[i] + b, h * group:(h + 1) * group].double().transpose(0, 1)
                s = (torch.matmul(q, k.t()) / math.sqrt(dim)).masked_fill(hidden, -math.inf)
                w = torch.softmax(s, -1).masked_fill(hidden.all(1)[None, :, None], 0.0)
                out[sq[i] + a:sq[i] + b, h * group:(h + 1) * group] = torch.matmul(w, v).transpose(0, 1)
    return out


# ------------------------------------------------------------------------------------------------------------ the work
def work(case):
    op, dim, kv = case["op"], case["dim"], case["kv_heads"]
    per_token = lambda kind: 2 * kv * (dim * _SIZE[kind] + (0 if kind == "bf16" else 4))    # a token's keys and values in the cache
    if op in ("rotate", "write"):
        tokens, x = case["tokens"], _SIZE[case["x"]]
        stored = 0 if case["cache"] == "none" else tokens * (per_token(case["cache"]) + 4)
        if op == "write":
            return dict(bytes=tokens * 2 * kv * dim * x + stored, flops=6 * tokens * kv * dim)
        qh, dense = case["q_heads"], case["cache"] == "none"
        read = tokens * ((qh + (1 if dense else 2) * kv) * dim * x + 4 + 4 * case["rotary"])
        return dict(bytes=read + 2 * tokens * (qh + (kv if dense else 0)) * dim + stored, flops=10 * tokens * (qh + kv) * dim)
    lengths = _lengths(case)
    if op == "read":
        total = sum(lengths)
        return dict(bytes=total * (per_token(case["cache"]) + 2 * kv * dim * _SIZE[case["x"]]), flops=2 * total * kv * dim)
    qh = case["q_heads"]
    if op == "token":
        seen = sum(min(n, case["window"]) if case["window"] else n for n in lengths)
        return dict(bytes=seen * per_token(case["cache"]) + 4 * case["seqs"] * qh * dim, flops=4 * seen * qh * dim)
    pairs = 0
    for n in lengths:
        m = n + case["prefix"]
        if not case["causal"] and not case["window"]:
            pairs += n * m
            continue
        for i in range(n):                                   # row i sees columns up to `last`, and no more than its window
            last = min(m, i + m - n + 1) if case["causal"] else m
            first = max(0, i + m - n + 1 - case["window"]) if case["window"] else 0
            pairs += max(0, last - first)
    total = sum(lengths)
    return dict(bytes=4 * total * qh * dim + 4 * (total + case["seqs"] * case["prefix"]) * kv * dim, flops=4 * pairs * qh * dim)
