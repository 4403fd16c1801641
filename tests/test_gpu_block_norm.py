"""The block norm and its backward pass against the definition in 64 bits: kinds, gates, types, odd sizes, pitches and
alignments, single rows, rows that hold NaN, output as operands of the 8-bit products; gradients against autograd of the
definition and against differences; refusals.

Tolerances.  A row sum of n terms is added in blocks of 8 or more per thread and then pairwise: its relative error
is below (8 * 4 + 10) * 2^-24 < 2^-18 of the sum of magnitudes, so a standardised value v is off by at most
2^-18 * (|v| + max|row| * inv) (the second part from the mean of a layer norm), and each norm, product and sum after it
adds a few 2^-24.  F = 2^-16 on the magnitudes that are added up covers two norms in a row; a result in bf16 (8 bits of
significand) is rounded by another 2^-8 of itself at most."""
import itertools

import numpy as np
import pytest
import torch

import paper_2506_17870_b200 as nq
from fp8_reference import block_norm, quantize

pytestmark = pytest.mark.gpu
NONE, RMS, LAYER = 0, 1, 2
F = 2.0 ** -16
TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16)]


def ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 0.0


def near(got, want, size):
    """|got - want| <= F * size + the rounding of got's type; size: float64, magnitudes that were added up."""
    rounding = ulp(got.dtype)
    got, want = got.double().cpu(), want.double()
    err = (got - want).abs()
    tol = F * size + rounding * want.abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-300)).max())


def make(rows, cols, tx, ty, gate=None, group=0, post=RMS, pre=RMS, bias=True, block=True, seed=0, mean=0.0):
    g = torch.Generator().manual_seed(rows * 7919 + cols + seed)
    n = lambda *s: torch.randn(*s, generator=g)
    st = dict(x=(n(rows, cols) + mean).to(tx).cuda(), y=(0.5 * n(rows, cols) + mean).to(ty).cuda() if block else None)
    vec = lambda on, c: (c + 0.3 * n(cols)).cuda() if on else None
    st.update(post=post if block else NONE, pre=pre, skip_scale=0.9, branch_scale=0.7, eps=1e-5, rows_per_gate=group,
              post_weight=vec(block and post, 1.0), post_bias=vec(block and post and bias, 0.0), pre_weight=vec(pre, 1.0),
              pre_bias=vec(pre and bias, 0.0), gate=None)
    if block and gate is not None:
        st["gate"] = (0.6 + 0.3 * n(-(-rows // group) if group else 1, cols)).cuda()
    return st


def split(st):
    st = dict(st)
    return st.pop("x"), st.pop("y"), st


def expected(st):
    d = lambda t: None if t is None else t.double().cpu()
    return block_norm(d(st["x"]), d(st["y"]), st["post"], d(st["post_weight"]), d(st["post_bias"]), d(st["gate"]), st["rows_per_gate"],
                      st["skip_scale"], st["branch_scale"], st["pre"], d(st["pre_weight"]), d(st["pre_bias"]), st["eps"])


def sizes(st, r):
    """Magnitudes behind r and h (a row's largest value stands for the sums over it)."""
    top = lambda t: t.abs().max(1, keepdim=True).values
    y = st["y"].double().cpu() if st["y"] is not None else torch.zeros_like(r)
    size_r = r.abs() + st["x"].double().cpu().abs() + 1.0
    if st["post"] != NONE:
        sd = torch.sqrt(((y - (y.mean(1, keepdim=True) if st["post"] == LAYER else 0)) ** 2).mean(1, keepdim=True) + st["eps"])
        size_r = size_r + 3 * top(y) / sd
    else:
        size_r = size_r + 3 * y.abs()
    sd = torch.sqrt(((r - (r.mean(1, keepdim=True) if st["pre"] == LAYER else 0)) ** 2).mean(1, keepdim=True) + st["eps"])
    size_h = 1.0 + 3 * (top(size_r) / sd + top(r) / sd)
    return size_r, size_h


def check(st, h_dtype=None, **more):
    x, y, how = split(st)
    r, h, hs = nq.nq_block_norm(x, y, h_dtype=h_dtype, **how, **more)
    want_r, want_h = expected(st)
    size_r, size_h = sizes(st, want_r)
    if r is not None:
        near(r, want_r, size_r)
    if st["pre"] != NONE:
        near(h, want_h, size_h)
    else:
        assert h is None
    return r, h


SHAPES = [(1, 1), (3, 7), (2, 8), (5, 31), (9, 256), (4, 264), (7, 768), (33, 100), (2, 2048), (3, 1138), (2, 4096), (3, 4097), (2, 5000),
          (2, 8192), (1, 9000), (2, 16384)]


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(rows, cols, tx, ty):
    check(make(rows, cols, tx, ty, gate=True))
    check(make(rows, cols, tx, ty, post=LAYER, pre=LAYER, seed=1))


@pytest.mark.parametrize("post,pre", [p for p in itertools.product((NONE, RMS, LAYER), repeat=2)])
@pytest.mark.parametrize("gate,group", [(None, 0), (True, 0), (True, 1), (True, 3), (True, 50)])
@pytest.mark.parametrize("bias", [False, True])
def test_kinds_and_gates(post, pre, gate, group, bias):
    check(make(11, 328, torch.float32, torch.bfloat16, gate, group, post, pre, bias))


@pytest.mark.parametrize("pre", [RMS, LAYER])
def test_plain_norm_of_the_stream(pre):
    st = make(6, 500, torch.float32, torch.float32, pre=pre, block=False)
    r, _ = check(st)
    assert r is None
    r, _ = check(st, want_r=True)
    assert r is not None


def test_large_mean():
    """The variance comes from centred values: a mean of 1000 deviations costs 1000 * 2^-24 and no more."""
    st = make(4, 4096, torch.float32, torch.float32, post=LAYER, pre=LAYER, mean=1000.0)
    check(st)


@pytest.mark.parametrize("cols,pitch,offset", [(256, 264, 8), (256, 257, 0), (256, 256, 1), (250, 256, 0), (4096, 4100, 4)])
@pytest.mark.parametrize("tx,ty", TYPES)
def test_pitch_and_alignment(cols, pitch, offset, tx, ty):
    st = make(5, cols, tx, ty, gate=True)
    for name in ("x", "y"):
        buf = torch.full((5 * pitch + offset + 16,), 1e3, dtype=st[name].dtype, device="cuda")
        v = buf[offset:offset + 5 * pitch].view(5, pitch)[:, :cols]
        v.copy_(st[name])
        st[name] = v
    check(st)
    want = expected(st)[0]
    x, y, how = split(st)
    r, _, _ = nq.nq_block_norm(x, y, r_out=x, **how)                       # in place
    assert r.data_ptr() == x.data_ptr()
    near(x, want, sizes({**st, "x": want}, want)[0] + 2 * want.abs())


@pytest.mark.parametrize("rows,cols", [(1, 4096), (5, 768), (3, 1138), (2, 130), (4, 8192), (3, 100), (1, 16384)])
@pytest.mark.parametrize("tx,ty", TYPES)
def test_e4m3_operand(rows, cols, tx, ty):
    """Codes and scales are the quantiser's, of an h that is off by the norm's fp32 error: a code may fall to a
    neighbour's (one step of e4m3 is at most 1/8 of the value, or 2^-9 below 2^-6), never further."""
    st = make(rows, cols, tx, ty, gate=True, pre=LAYER)
    x, y, how = split(st)
    r, h, hs = nq.nq_block_norm(x, y, h_dtype=torch.float8_e4m3fn, **how)
    want_r, want_h = expected(st)
    near(r, want_r, sizes(st, want_r)[0])
    q, s = quantize(want_h.float().numpy(), 1)
    size_h = float(sizes(st, want_r)[1].max())
    got_s = hs.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got_s - s) <= (F * size_h / 448 + 1e-7 * s))
    got = h.float().cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - q) <= np.maximum(np.abs(q) / 8 * 1.0001, 2.0 ** -9 * 1.0001))
    assert np.mean(got != q) < 0.01


@pytest.mark.parametrize("cols", [768, 1138, 24])
def test_int8_operand(cols):
    st = make(9, cols, torch.float32, torch.bfloat16)
    x, y, how = split(st)
    _, h, hs = nq.nq_block_norm(x, y, h_dtype=torch.int8, h_scale=0.02, **how)
    want_r, want_h = expected(st)
    v = want_h / float(np.float32(0.02))
    off = F * sizes(st, want_r)[1] / 0.02
    assert hs is None
    q = h.double().cpu()
    assert bool((q >= torch.clamp(torch.round(v - off), -128, 127)).all() and (q <= torch.clamp(torch.round(v + off), -128, 127)).all())


def test_nan_stays_in_its_row():
    st = make(6, 640, torch.float32, torch.float32, post=LAYER)
    st["x"][2, 5] = float("nan")
    st["y"][4, 600] = float("inf")
    x, y, how = split(st)
    r, h, _ = nq.nq_block_norm(x, y, **how)
    bad = torch.isnan(h).all(1).cpu()
    assert bad.tolist() == [False, False, True, False, True, False]
    assert bool(torch.isnan(r[4]).all()) and int(torch.isnan(r[2]).sum()) == 1
    assert bool(torch.isfinite(h[[0, 1, 3, 5]]).all())


def test_zero_rows_of_values():
    """A row of zeros: rsqrt(eps) times zero."""
    x = torch.zeros(3, 512, device="cuda")
    _, h, _ = nq.nq_block_norm(x, None, pre=LAYER, eps=1e-6)
    assert bool((h == 0).all())
    _, h, hs = nq.nq_block_norm(x, None, pre=RMS, h_dtype=torch.float8_e4m3fn)
    assert bool((h.float() == 0).all()) and bool((hs == 2.0 ** -126).all())


# ----------------------------------------------------------------------------------------------------------- backward
def gradients(st, dr, dh):
    """autograd of the definition in 64 bits, at the r that the forward pass stored."""
    d = lambda t: None if t is None else t.double().cpu().requires_grad_(True)
    r, y = d(st["r"]), d(st["y"])
    pw, pb, gate, qw, qb = (d(st[k]) for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias"))
    _, h = block_norm(r, None, 0, None, None, None, 0, 1.0, 1.0, st["pre"], qw, qb, st["eps"])
    loss = 0.0
    if dh is not None:
        loss = loss + (h * dh.double().cpu()).sum()
    if dr is not None:
        loss = loss + (r * dr.double().cpu()).sum()
    leaves = [r] + ([t for t in (qw, qb) if t is not None] if st["pre"] else [])
    got = dict(zip(("r", "qw", "qb") if qb is not None else ("r", "qw"), torch.autograd.grad(loss, leaves)))
    g = got["r"]
    branch = None
    if y is not None:
        zero = torch.zeros_like(g)
        b, _ = block_norm(zero, y, st["post"], pw, pb, gate, st["rows_per_gate"], 0.0, st["branch_scale"], 0, None, None, st["eps"])
        names = [n for n, t in (("y", y), ("pw", pw), ("pb", pb), ("gate", gate)) if t is not None]
        branch = dict(zip(names, torch.autograd.grad((b * g).sum(), [t for t in (y, pw, pb, gate) if t is not None])))
        got.update(branch)
    got["x"] = st["skip_scale"] * g
    return got


def backward_case(rows, cols, tx, ty, **how):
    st = make(rows, cols, tx, ty, **how)
    g = torch.Generator().manual_seed(5)
    r = expected(st)[0].to(tx)
    st["r"] = r.cuda()
    dr = torch.randn(rows, cols, generator=g).to(tx).cuda()
    dh = torch.randn(rows, cols, generator=g).to(ty).cuda() if st["pre"] else None
    return st, dr, dh


def run_backward(st, dr, dh):
    how = {k: v for k, v in st.items() if k not in ("x", "y", "r")}
    return nq.nq_block_norm_backward(st["r"], st["y"], dr=dr, dh=dh, **how)


def check_backward(st, dr, dh):
    """Row gradients within F of the row's largest magnitudes (times the inverse deviations, which the inputs keep near or below
    4), sums over rows within F of the sum of magnitudes, estimated by rows * 8."""
    want = gradients(st, dr, dh)
    dx, dy, dgate, dpw, dpb, dqw, dqb = run_backward(st, dr, dh)
    top = lambda t: t.abs().max(1, keepdim=True).values + 8.0
    near(dx, want["x"], top(want["x"]) * 8)
    rows = dx.shape[0]
    for got, name in ((dy, "y"), (dgate, "gate"), (dpw, "pw"), (dpb, "pb"), (dqw, "qw"), (dqb, "qb")):
        assert (got is None) == (name not in want), name
        if got is None:
            continue
        near(got, want[name], top(want["y"]) * 8 if name == "y" else torch.full_like(want[name], 8.0 * rows ** 0.5 + 8 * float(want[name].abs().max())))
    again = run_backward(st, dr, dh)
    for a, b in zip((dx, dy, dgate, dpw, dpb, dqw, dqb), again):
        assert a is None and b is None or torch.equal(a, b)                  # sums are joined in a fixed order


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 31), (40, 256), (700, 264), (7, 768), (900, 100), (5, 1138), (300, 2048), (6, 4096), (3, 5000), (2, 8192), (2, 16384)])
def test_backward_shapes(rows, cols, tx, ty):
    check_backward(*backward_case(rows, cols, tx, ty, gate=True))
    check_backward(*backward_case(rows, cols, tx, ty, post=LAYER, pre=LAYER, gate=True, group=max(1, rows // 3)))


@pytest.mark.parametrize("post,pre", [p for p in itertools.product((NONE, RMS, LAYER), repeat=2)])
@pytest.mark.parametrize("gate,group", [(None, 0), (True, 0), (True, 1), (True, 7), (True, 5000)])
@pytest.mark.parametrize("bias", [False, True])
def test_backward_kinds_and_gates(post, pre, gate, group, bias):
    check_backward(*backward_case(61, 328, torch.float32, torch.float32, post=post, pre=pre, gate=gate, group=group, bias=bias))


def test_backward_parts():
    st, dr, dh = backward_case(20, 264, torch.float32, torch.float32, gate=True)
    check_backward(st, None, dh)
    st, dr, dh = backward_case(20, 264, torch.bfloat16, torch.bfloat16, block=False)
    check_backward(st, dr, dh)
    check_backward(st, None, dh)


@pytest.mark.parametrize("pitch,offset", [(272, 0), (265, 0), (264, 1)])
def test_backward_pitch_and_alignment(pitch, offset):
    st, dr, dh = backward_case(30, 264, torch.float32, torch.bfloat16, gate=True, post=LAYER)

    def put(t):
        buf = torch.full((30 * pitch + offset,), 1e3, dtype=t.dtype, device="cuda")
        v = buf[offset:].view(30, pitch)[:, :264]
        v.copy_(t)
        return v
    st["r"], st["y"] = put(st["r"]), put(st["y"])
    check_backward(st, put(dr), put(dh))


def test_backward_against_differences():
    """<gradient, direction> against central differences of the forward pass in 64 bits; differences of step 1e-5
    are off by about 1e-10, so F times the number of terms' root is the kernel's part."""
    rows, cols = 24, 200
    st, _, dh = backward_case(rows, cols, torch.float32, torch.float32, post=LAYER, pre=RMS, gate=True, group=6)
    d = lambda t: t.double().cpu()
    dr = torch.randn(rows, cols, generator=torch.Generator().manual_seed(9))
    names = ("x", "y", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias")
    base = {n: d(st[n]) for n in names}

    def loss(p):
        r, h = block_norm(p["x"], p["y"], st["post"], p["post_weight"], p["post_bias"], p["gate"], 6, st["skip_scale"], st["branch_scale"],
                          st["pre"], p["pre_weight"], p["pre_bias"], st["eps"])
        return (r * dr.double()).sum() + (h * d(dh)).sum()
    got = run_backward(st, dr.cuda(), dh)
    for i, n in enumerate(names):
        way = torch.randn(base[n].shape, generator=torch.Generator().manual_seed(20 + i), dtype=torch.float64)
        eps = 1e-5
        diff = (loss({**base, n: base[n] + eps * way}) - loss({**base, n: base[n] - eps * way})) / (2 * eps)
        mine = (got[i].double().cpu() * way).sum()
        assert abs(float(mine - diff)) <= 64 * F * (rows * cols) ** 0.5, n


def test_no_rows():
    z = torch.empty(0, 64, device="cuda")
    r, h, _ = nq.nq_block_norm(z, z)
    assert r.shape == h.shape == (0, 64)
    w = torch.ones(64, device="cuda")
    got = nq.nq_block_norm_backward(z, z, dr=z, dh=z, pre_weight=w, post=RMS, post_weight=w, gate=torch.ones(1, 64, device="cuda"))
    assert bool((got[2] == 0).all() and (got[3] == 0).all() and (got[5] == 0).all())


def test_other_stream():
    st = make(64, 4096, torch.bfloat16, torch.bfloat16, gate=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        st["x"] = st["x"] * 2
        x, y, how = split(st)
        r, h, _ = nq.nq_block_norm(x, y, **how)
    side.synchronize()
    want_r, want_h = expected(st)
    near(r, want_r, sizes(st, want_r)[0])
    near(h, want_h, sizes(st, want_r)[1])


def test_refusals():
    x, b = torch.zeros(8, 32, device="cuda"), torch.zeros(8, 32, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(32, device="cuda")
    bad = [dict(x=b, y=x), dict(x=x.half()), dict(x=x, y=x[:4]), dict(x=x, post=3), dict(x=x, y=x, post_weight=w[:16], post=RMS),
           dict(x=x, y=x, gate=w), dict(x=x, y=x, gate=w[None], rows_per_gate=4), dict(x=x, pre_weight=w.cpu()), dict(x=x.t()),
           dict(x=x, pre_weight=w.double()), dict(x=x, h_dtype=torch.float16), dict(x=x, y=x, rows_per_gate=-1), dict(x=x.cpu()),
           dict(x=x, r_out=b)]
    for k in bad:
        with pytest.raises(ValueError):
            nq.nq_block_norm(**k)
    refused = [dict(x=x, post=RMS), dict(x=x, gate=w[None]), dict(x=x, y=x, post_weight=w), dict(x=x, y=x, pre=NONE, pre_weight=w),
               dict(x=x, h_dtype=torch.int8, h_scale=0.0), dict(x=x, pre=NONE), dict(x=x, eps=-1.0),
               dict(x=torch.zeros(1, 16385, device="cuda"))]
    for k in refused:
        with pytest.raises(nq.NqError):
            nq.nq_block_norm(**k)
    for k in [dict(r=x), dict(r=x, pre=NONE), dict(r=x, dh=x, y=b), dict(r=x, dh=x, dr=b), dict(r=x, dr=x, dh=x, pre=NONE)]:
        with pytest.raises(ValueError):
            nq.nq_block_norm_backward(**k)
    for k in [dict(r=x, dh=x, post=RMS), dict(r=x, dh=x, gate=w[None]), dict(r=x, y=x, dh=x, post_weight=w),
              dict(r=x, dh=x, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))]:
        with pytest.raises(nq.NqError):
            nq.nq_block_norm_backward(**k)


# ------------------------------------------------------------------------------------- many rows to a thread block
def test_many_rows_layouts():
    """Enough rows that blocks work through many of them (rows ahead of the one in work are then in flight), of few, of
    whole and of uneven numbers of pieces a thread; against the definition in 64 bits on the device."""
    for rows, cols, tx, ty, kind, group in ((9001, 512, torch.bfloat16, torch.bfloat16, RMS, 0), (9001, 768, torch.float32, torch.bfloat16, LAYER, 197),
                                            (5003, 1032, torch.float32, torch.float32, LAYER, 0), (3001, 4096, torch.bfloat16, torch.bfloat16, RMS, 1),
                                            (2003, 4104, torch.float32, torch.bfloat16, LAYER, 500), (1501, 8192, torch.bfloat16, torch.bfloat16, RMS, 0),
                                            (901, 12000, torch.bfloat16, torch.bfloat16, LAYER, 0), (5001, 264, torch.bfloat16, torch.bfloat16, LAYER, 3)):
        st = make(rows, cols, tx, ty, gate=True, group=group, post=kind, pre=kind)
        check(st)
        if rows * cols <= 9001 * 768:
            st["post"], st["post_weight"], st["post_bias"] = NONE, None, None
            check(st, h_dtype=torch.float32)
            check(make(rows, cols, tx, tx, post=NONE, pre=kind, block=False))


@pytest.mark.parametrize("rows,cols,tx,ty,kind,group", [
    (9001, 512, torch.bfloat16, torch.bfloat16, RMS, 0), (9001, 768, torch.float32, torch.bfloat16, LAYER, 197),
    (4003, 1032, torch.float32, torch.float32, LAYER, 0), (3001, 4096, torch.bfloat16, torch.bfloat16, RMS, 1),
    (1003, 4104, torch.float32, torch.bfloat16, LAYER, 500), (1501, 8192, torch.bfloat16, torch.bfloat16, RMS, 0),
    (901, 12000, torch.bfloat16, torch.bfloat16, LAYER, 0)])
def test_many_rows_backward(rows, cols, tx, ty, kind, group):
    check_backward(*backward_case(rows, cols, tx, ty, post=kind, pre=kind, gate=True, group=group))


@pytest.mark.parametrize("cols,pitch,offset", [(768, 771, 1), (1001, 1001, 0), (1138, 1140, 3), (4097, 4097, 0)])
@pytest.mark.parametrize("tx,ty", TYPES)
def test_many_rows_that_start_anywhere(cols, pitch, offset, tx, ty):
    rows = 4500 if cols < 2000 else 1500

    def put(t):
        buf = torch.full((rows * pitch + offset,), 1e3, dtype=t.dtype, device="cuda")
        v = buf[offset:].view(rows, pitch)[:, :cols]
        v.copy_(t)
        return v
    st, dr, dh = backward_case(rows, cols, tx, ty, gate=True, post=LAYER, group=700)
    for name in ("x", "y", "r"):
        st[name] = put(st[name])
    forward = {k: v for k, v in st.items() if k != "r"}
    check(forward)
    check_backward(st, put(dr), put(dh))


def test_many_rows_backward_without_post_norm():
    check_backward(*backward_case(6001, 768, torch.float32, torch.bfloat16, post=NONE, pre=LAYER, gate=True, group=100))
    st, dr, dh = backward_case(6001, 768, torch.bfloat16, torch.bfloat16, post=NONE, pre=RMS, block=False)
    check_backward(st, dr, dh)
