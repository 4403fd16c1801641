"""Cases of the low-precision linear operators: the e4m3 quantiser with a scale for each 128 values, the product of
e4m3 matrices with a scale for each block of 128, and the norms before and after a block with its gate and residual
scale, forward and backward.

Layouts.  An e4m3 matrix is [rows, cols] with a row pitch that is a multiple of 16 bytes.  Its scales are fp32,
groups first: [ceil(cols / 128), rows] for groups of 1 x 128, [ceil(cols / 128), ceil(rows / 128)] for blocks of
128 x 128.  A value is its e4m3 number times its group's scale.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
_SIZE = {"bf16": 2, "f32": 4, "fp8": 1, "int8": 1}
_E4M3_MAX = 448.0
_EPS = 1e-6


def _up(v, m):
    return -(-v // m) * m


# ----------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # activations of five tokens being generated, ahead of a product: all latency
        dict(name="quantise 5 tokens", op="quantize", rows=5, cols=4096, block_rows=1, dtype="bf16", sides="row"),
        # a training batch's activations: once for the forward product, once transposed for the weight gradient
        dict(name="quantise batch both ways", op="quantize", rows=16384, cols=8192, block_rows=1, dtype="bf16", sides="both"),
        # a layer's fp32 master weights after an optimiser step, for the forward and the input-gradient product
        dict(name="quantise weights", op="quantize", rows=8192, cols=4096, block_rows=128, dtype="f32", sides="both"),
        # one generated token: the weights are read once
        dict(name="product 1 token", op="gemm", m=1, n=4096, k=4096, b_block_rows=128, out="bf16", bias=False),
        # a few dozen sequences that generate together, odd in number
        dict(name="product 37 tokens", op="gemm", m=37, n=8192, k=4096, b_block_rows=128, out="bf16", bias=True),
        # the fused qkv linear of the repository's image transformer on 64 images of 197 tokens
        dict(name="product 64 images qkv", op="gemm", m=12608, n=2304, k=768, b_block_rows=128, out="bf16", bias=True),
        # weight gradient over 12608 tokens (98.5 groups): both operands transposed, fp32 out
        dict(name="product weight gradient", op="gemm", m=4096, n=4096, k=12608, b_block_rows=1, out="f32", bias=False),
        # the repository's middle square product
        dict(name="product 8192", op="gemm", m=8192, n=8192, k=8192, b_block_rows=128, out="bf16", bias=False),
        # between two blocks while five tokens are generated; the next product's operand comes out quantised
        dict(name="norm 5 tokens", op="norm", rows=5, cols=4096, kind="rms", post=True, gate="channel", group=0, stream="bf16", branch="bf16", h="fp8"),
        # the same over a long prompt or a training batch
        dict(name="norm long batch", op="norm", rows=16384, cols=8192, kind="rms", post=True, gate="channel", group=0, stream="bf16", branch="bf16", h="fp8"),
        # backward of the image transformer's norms: fp32 stream, a gate for each of 64 images
        dict(name="norm gradient 64 images", op="norm_grad", rows=12608, cols=768, kind="layer", post=True, gate="group", group=197, stream="f32", branch="bf16"),
        # backward over a training batch of a wider model
        dict(name="norm gradient long batch", op="norm_grad", rows=16384, cols=4096, kind="rms", post=True, gate="channel", group=0, stream="bf16", branch="bf16"),
    ]


def _size(rng, low, high):
    """A size spread evenly over its logarithm; half of them as they fall, half rounded up to a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return v if rng.random() < 0.5 else max(low, min(high, _up(v, 64)))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "norm", "norm_grad"])
    if op == "gemm":
        grad = rng.random() < 0.3
        m, n, k = _size(rng, 64 if grad else 1, 16384), _size(rng, 64, 16384), _size(rng, 64, 16384)
        while m * n * k > 8192 ** 3:
            m, n, k = -(-m // 2), -(-n // 2), -(-k // 2)
        return dict(op=op, m=m, n=n, k=k, b_block_rows=1 if grad else 128, out=rng.choice(["bf16", "f32"]), bias=not grad and rng.random() < 0.5)
    rows, cols = _size(rng, 1, 50432), _size(rng, 64, 8192)
    most = 16384 * (4096 if op == "norm_grad" else 8192)
    while rows * cols > most:
        rows = -(-rows // 2)
    if op == "quantize":
        return dict(op=op, rows=rows, cols=cols, block_rows=rng.choice([1, 128]), dtype=rng.choice(["bf16", "f32"]), sides=rng.choice(["row", "both"]))
    gate = rng.choice(["none", "channel", "group"])
    stream, branch = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
    case = dict(op=op, rows=rows, cols=cols, kind=rng.choice(["rms", "layer"]), post=rng.random() < 0.7, gate=gate,
                group=_size(rng, 1, max(2, rows)) if gate == "group" else 0, stream=stream, branch=branch)
    if stream == "f32":
        while case["rows"] * cols > most // 2:
            case["rows"] = -(-case["rows"] // 2)
    if op == "norm":
        case["h"] = rng.choice([branch, "fp8", "fp8", "int8"])
    return case


# ---------------------------------------------------------------------------------------------------------- the inputs
class _Make:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def activations(self, rows, cols):
        """Normal values whose channels differ in size, a few of them much larger, as hidden states are."""
        c = torch.exp(0.5 * self.normal(cols))
        return self.normal(rows, cols) * torch.where(torch.rand(cols, generator=self.g, device="cuda") < 0.005, 12.0 * c, c)


def _pitched(q):
    """The same matrix with a row pitch that is a multiple of 16."""
    rows, cols = q.shape
    buf = torch.zeros(rows, _up(cols, 16), dtype=torch.uint8, device=q.device)
    buf[:, :cols] = q.view(torch.uint8)
    return buf.view(torch.float8_e4m3fn)[:, :cols]


def prepare(case, seed):
    make = _Make(seed)
    st = dict(case=case)
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        x = make.activations(rows, cols) if case["block_rows"] == 1 else make.normal(rows, cols) / math.sqrt(cols)
        st["x"] = x.to(_TYPES[case["dtype"]])
    elif case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        a, st["sa"] = _plain_quantize(make.activations(m, k), 1)
        b, st["sb"] = _plain_quantize(make.normal(n, k) / math.sqrt(k), case["b_block_rows"])
        st["a"], st["b"] = _pitched(a), _pitched(b)
        st["bias"] = make.normal(n) if case["bias"] else None
    else:
        rows, cols, layer = case["rows"], case["cols"], case["kind"] == "layer"
        weight = lambda: 1.0 + 0.2 * make.normal(cols)
        stream, branch = _TYPES[case["stream"]], _TYPES[case["branch"]]
        st["x"] = make.activations(rows, cols).to(stream)
        st["y"] = (0.3 * make.activations(rows, cols)).to(branch)
        st["gate"] = {"none": lambda: None, "channel": lambda: 0.5 + 0.2 * make.normal(1, cols),
                      "group": lambda: 0.5 + 0.2 * make.normal(-(-rows // max(1, case["group"])), cols)}[case["gate"]]()
        st["post_weight"] = weight() if case["post"] else None
        st["post_bias"] = 0.1 * make.normal(cols) if case["post"] and layer else None
        st["pre_weight"], st["pre_bias"] = weight(), 0.1 * make.normal(cols) if layer else None
        st["skip"], st["branch"] = 0.9, 0.7
        st["h_scale"] = 0.05                       # static activation scale of an INT8 hand-over
        if case["op"] == "norm_grad":              # what the forward pass left, and the gradients that arrive
            st["r"] = _plain_norm(st)[0]
            del st["x"]
            st["dr"], st["dh"] = make.normal(rows, cols).to(stream), make.normal(rows, cols).to(branch)
    return st


# ------------------------------------------------------------------------------------------------------- the operators
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        if op == "quantize":
            q, s = _plain_quantize(st["x"], case["block_rows"])
            return (q, s) if case["sides"] == "row" else (q, s) + _plain_quantize(st["x"].t(), case["block_rows"])
        if op == "gemm":
            return _plain_gemm(st)
        if op == "norm":
            r, h = _plain_norm(st)
            if case["h"] == "fp8":
                return (r,) + _plain_quantize(h, 1)
            if case["h"] == "int8":
                q = torch.clamp(torch.round(h * (1.0 / st["h_scale"])), -128, 127).to(torch.int8)
                return r, q.to(torch.bfloat16) * st["h_scale"]
            return r, h.to(_TYPES[case["h"]])
        return _plain_norm_grad(st)
    import paper_2506_17870_b200 as nq
    if op == "quantize":
        q, s, qt, t = nq.nq_fp8_quantize(st["x"], block_rows=case["block_rows"], transposed=case["sides"] == "both")
        return (q, s) if qt is None else (q, s, qt, t)
    if op == "gemm":
        return nq.nq_fp8_gemm(st["a"], st["sa"], st["b"], st["sb"], b_block_rows=case["b_block_rows"], bias=st["bias"], y_dtype=_TYPES[case["out"]])
    kind = nq.NQ_NORM_LAYER if case["kind"] == "layer" else nq.NQ_NORM_RMS
    how = dict(post=kind if case["post"] else nq.NQ_NORM_NONE, post_weight=st["post_weight"], post_bias=st["post_bias"], gate=st["gate"],
               rows_per_gate=case["group"], skip_scale=st["skip"], branch_scale=st["branch"], pre=kind, pre_weight=st["pre_weight"],
               pre_bias=st["pre_bias"], eps=_EPS)
    if op == "norm":
        r, h, s = nq.nq_block_norm(st["x"], st["y"], h_dtype=_TYPES[case["h"]], h_scale=st["h_scale"], **how)
        return (r, h, s) if case["h"] == "fp8" else (r, h.to(torch.bfloat16) * st["h_scale"]) if case["h"] == "int8" else (r, h)
    return nq.nq_block_norm_backward(st["r"], st["y"], dr=st["dr"], dh=st["dh"], **how)


# -------------------------------------------------------------------------------------------------------- plain forms
def _plain_quantize(x, block_rows):
    """x [rows, cols] -> e4m3 [rows, cols] and its scales, groups first."""
    rows, cols = x.shape
    f = torch.zeros(_up(rows, block_rows), _up(cols, 128), dtype=torch.float32, device=x.device)
    f[:rows, :cols] = x
    f = f.view(f.shape[0] // block_rows, block_rows, f.shape[1] // 128, 128)
    s = torch.clamp(f.abs().amax(dim=(1, 3)) / _E4M3_MAX, min=2.0 ** -126)
    q = torch.clamp(f * (1.0 / s)[:, None, :, None], -_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(_up(rows, block_rows), _up(cols, 128))[:rows, :cols], s.t().contiguous()


def _spread(s, block_rows, rows, cols):
    """Scales, groups first -> one for each value [rows, cols]."""
    return s.repeat_interleave(block_rows, 1)[:, :rows].t().repeat_interleave(128, 1)[:, :cols]


def _plain_gemm(st):
    case = st["case"]
    a = st["a"].float() * _spread(st["sa"], 1, case["m"], case["k"])
    b = st["b"].float() * _spread(st["sb"], case["b_block_rows"], case["n"], case["k"])
    y = a @ b.t()
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(_TYPES[case["out"]])


def _standard(v, layer):
    """The row's values without their mean (layer) over their root mean square, and that root's inverse."""
    if layer:
        v = v - v.mean(dim=1, keepdim=True)
    inv = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + _EPS)
    return v * inv, inv


def _gates(st):
    case = st["case"]
    if case["gate"] == "none":
        return 1.0
    return st["gate"] if case["gate"] == "channel" else st["gate"].repeat_interleave(case["group"], 0)[: case["rows"]]


def _plain_norm(st):
    """(r in the stream's type, h in 32 bits)"""
    case = st["case"]
    layer = case["kind"] == "layer"
    u = st["y"].float()
    if case["post"]:
        u = _standard(u, layer)[0] * st["post_weight"]
        if layer:
            u = u + st["post_bias"]
    r = st["skip"] * st["x"].float() + st["branch"] * _gates(st) * u
    h = _standard(r, layer)[0] * st["pre_weight"]
    if layer:
        h = h + st["pre_bias"]
    return r.to(_TYPES[case["stream"]]), h


def _plain_back(w, v, inv, d, layer):
    """Gradient of a norm's input from its standardised values v, and of its weight and bias."""
    wd = d * w
    g = wd - v * (wd * v).mean(dim=1, keepdim=True)
    if layer:
        g = g - wd.mean(dim=1, keepdim=True)
    return g * inv, (d * v).sum(dim=0), d.sum(dim=0) if layer else None


def _plain_norm_grad(st):
    case = st["case"]
    layer, rows = case["kind"] == "layer", case["rows"]
    v, inv = _standard(st["r"].float(), layer)
    g, dpre_weight, dpre_bias = _plain_back(st["pre_weight"], v, inv, st["dh"].float(), layer)
    g = g + st["dr"].float()
    dx = (st["skip"] * g).to(_TYPES[case["stream"]])
    u = st["y"].float()
    if case["post"]:
        v, inv = _standard(u, layer)
        u = v * st["post_weight"]
        if layer:
            u = u + st["post_bias"]
    dgate = None
    if case["gate"] == "channel":
        dgate = (st["branch"] * u * g).sum(dim=0, keepdim=True)
    elif case["gate"] == "group":
        each = torch.zeros(len(st["gate"]) * case["group"], case["cols"], device=g.device)
        each[:rows] = st["branch"] * u * g
        dgate = each.view(-1, case["group"], case["cols"]).sum(dim=1)
    du = st["branch"] * _gates(st) * g
    dpost_weight = dpost_bias = None
    dy = du
    if case["post"]:
        dy, dpost_weight, dpost_bias = _plain_back(st["post_weight"], v, inv, du, layer)
    return dx, dy.to(_TYPES[case["branch"]]), dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias


# --------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; in the place of numbers held in 8 bits, the values that
    are rounded to them."""
    st = prepare(case, seed)
    d = lambda name: st[name].double()
    if case["op"] == "quantize":
        def codes(x):
            parts, scales = [], []
            for c in x.split(128, dim=1):
                a = c.abs().amax(dim=1)
                if case["block_rows"] == 128:
                    a = torch.stack([p.max() for p in a.split(128)])
                s = a / 448
                scales.append(s)
                parts.append(c / (s if case["block_rows"] == 1 else s.repeat_interleave(128)[: len(c)])[:, None])
            return torch.cat(parts, 1), torch.stack(scales)
        x = d("x")
        return codes(x) if case["sides"] == "row" else codes(x) + codes(x.t())
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        y = torch.zeros(m, n, dtype=torch.float64, device="cuda") if st["bias"] is None else d("bias").expand(m, n).clone()
        sa, sb = d("sa"), d("sb")
        for kb in range(-(-k // 128)):
            part = slice(128 * kb, min(k, 128 * kb + 128))
            col = sb[kb] if case["b_block_rows"] == 1 else sb[kb].repeat_interleave(128)[:n]
            y.addmm_(st["a"][:, part].double() * sa[kb][:, None], (st["b"][:, part].double() * col[:, None]).t())
        return y
    layer, rows, cols = case["kind"] == "layer", case["rows"], case["cols"]
    group = torch.arange(rows, device="cuda") // case["group"] if case["gate"] == "group" else torch.zeros(rows, dtype=torch.int64, device="cuda")
    gate = torch.ones(1, cols, dtype=torch.float64, device="cuda") if st["gate"] is None else d("gate")

    def norm(t, w, b):                              # value, and its gradient as a function of the output's
        mu = t.sum(1, keepdim=True) / cols if layer else 0.0
        sd = torch.sqrt(((t - mu) ** 2).sum(1, keepdim=True) / cols + _EPS)
        z = (t - mu) / sd

        def back(g):
            e = g * w
            inner = e - z * ((e * z).sum(1, keepdim=True) / cols) - ((e.sum(1, keepdim=True) / cols) if layer else 0.0)
            return inner / sd, (g * z).sum(0), g.sum(0) if layer else None
        return z * w + (b if layer else 0.0), back

    bias = lambda name: d(name) if layer else None
    u, back_post = norm(d("y"), d("post_weight"), bias("post_bias")) if case["post"] else (d("y"), None)
    if case["op"] == "norm":
        r = st["skip"] * d("x") + st["branch"] * gate[group] * u
        h, _ = norm(r, d("pre_weight"), bias("pre_bias"))
        if case["h"] == "int8":
            return r, torch.clamp(h, -128 * st["h_scale"], 127 * st["h_scale"])
        if case["h"] != "fp8":
            return r, h
        s = torch.stack([c.abs().amax(1) / 448 for c in h.split(128, dim=1)])
        return r, h / s.t().repeat_interleave(128, 1)[:, :cols], s
    _, back_pre = norm(d("r"), d("pre_weight"), bias("pre_bias"))
    g, dpre_weight, dpre_bias = back_pre(d("dh"))
    g = g + d("dr")
    dgate = None
    if case["gate"] != "none":
        dgate = torch.zeros_like(gate).index_add_(0, group, st["branch"] * u * g)
    du = st["branch"] * gate[group] * g
    dy, dpost_weight, dpost_bias = back_post(du) if case["post"] else (du, None, None)
    return st["skip"] * g, dy, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias


# ------------------------------------------------------------------------------------------------------------ the work
def work(case):
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        sides = 1 if case["sides"] == "row" else 2
        scales = -(-cols // 128) * -(-rows // case["block_rows"]) + (sides - 1) * -(-rows // 128) * -(-cols // case["block_rows"])
        return dict(bytes=rows * cols * (_SIZE[case["dtype"]] + sides) + 4 * scales, flops=3 * sides * rows * cols)
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        groups = -(-k // 128)
        return dict(bytes=(m + n) * k + 4 * groups * (m + -(-n // case["b_block_rows"])) + m * n * _SIZE[case["out"]] + (4 * n if case["bias"] else 0),
                    flops=2 * m * n * k)
    rows, cols = case["rows"], case["cols"]
    stream, branch = _SIZE[case["stream"]], _SIZE[case["branch"]]
    vectors = (1 + case["post"]) * (2 if case["kind"] == "layer" else 1)
    gates = {"none": 0, "channel": 1, "group": -(-rows // max(1, case["group"]))}[case["gate"]]
    if case["op"] == "norm":
        scales = -(-cols // 128) * rows if case["h"] == "fp8" else 0
        return dict(bytes=rows * cols * (2 * stream + branch + _SIZE[case["h"]]) + 4 * scales + 4 * cols * (vectors + gates), flops=14 * rows * cols)
    # r, dr, y, dh in; dx, dy out; each parameter in and its gradient out (a bias is no input of its own gradient)
    return dict(bytes=rows * cols * (3 * stream + 3 * branch) + 8 * cols * (vectors + gates), flops=30 * rows * cols)
