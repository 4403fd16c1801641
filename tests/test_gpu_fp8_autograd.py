"""Autograd over the e4m3 entry points where a stack of RMS norms does not go: layer norms with biases, no pre norm, outputs of
another type than the branch, 8-bit outputs, second derivatives, weights that change after they were laid out.

Gradients have to be bit for bit those of nq_block_norm_backward on the r that the forward pass returned, and within the
bounds of test_gpu_block_norm.py (derived there) of 64-bit autograd of the definition."""
import copy

import pytest
import torch

import paper_2506_17870_b200 as nq
from paper_2506_17870_b200 import fp8_block as fb
from test_gpu_block_norm import F, LAYER, NONE, RMS, gradients, make, near

pytestmark = pytest.mark.gpu
PARAMS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")


def leaf(t):
    return None if t is None else t.detach().clone().requires_grad_(True)


def run(st, dr, dh, **more):
    """block_norm of the leaves and its backward pass -> (leaves, r, h)"""
    v = {k: leaf(st[k]) for k in ("x", "y") + PARAMS}
    how = {k: st[k] for k in ("post", "pre", "rows_per_gate", "skip_scale", "branch_scale", "eps")}
    r, h = fb.block_norm(v["x"], v["y"], v["post_weight"], v["gate"], v["pre_weight"], post_bias=v["post_bias"], pre_bias=v["pre_bias"], **how, **more)
    outs = [(r, dr)] + ([(h, dh)] if h is not None else [])
    torch.autograd.backward([o for o, _ in outs], [g for _, g in outs])
    return v, r, h


def check(st, v, r, dr, dh):
    """dh: as the entry point takes it"""
    how = {k: st[k] for k in ("post", "pre", "rows_per_gate", "skip_scale", "branch_scale", "eps") + PARAMS}
    got = nq.nq_block_norm_backward(r.detach(), st["y"], dr=dr, dh=dh, **how)
    names = ("x", "y", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias")
    for name, g in zip(names, got):
        if st[name] is None:
            assert g is None and v[name] is None
        else:
            assert v[name].grad is not None, f"{name} got no gradient"
            assert torch.equal(v[name].grad, g), name
    want = gradients({**st, "r": r.detach()}, dr, dh)
    rows = r.shape[0]
    top = lambda t: t.abs().max(1, keepdim=True).values + 8.0
    near(v["x"].grad, want["x"], top(want["x"]) * 8)
    for name, key in (("y", "y"), ("gate", "gate"), ("post_weight", "pw"), ("post_bias", "pb"), ("pre_weight", "qw"), ("pre_bias", "qb")):
        if st[name] is not None:
            near(v[name].grad, want[key], top(want["y"]) * 8 if key == "y" else torch.full_like(want[key], 8.0 * rows ** 0.5 + 8 * float(want[key].abs().max())))


def incoming(rows, cols, tr, th, seed=5):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(rows, cols, generator=g).to(tr).cuda(), torch.randn(rows, cols, generator=g).to(th).cuda()


@pytest.mark.parametrize("rows,cols,group", [(37, 264, 0), (394, 768, 197), (5, 31, 2)])
@pytest.mark.parametrize("tx,ty", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_layer_norm_biases(rows, cols, group, tx, ty):
    st = make(rows, cols, tx, ty, gate=True, group=group, post=LAYER, pre=LAYER)
    dr, dh = incoming(rows, cols, tx, ty)
    v, r, _ = run(st, dr, dh)
    check(st, v, r, dr, dh)


def test_bias_of_one_norm():
    for drop in ("post_bias", "pre_bias"):
        st = make(20, 264, torch.float32, torch.float32, gate=True, post=LAYER, pre=LAYER)
        st[drop] = None
        dr, dh = incoming(20, 264, torch.float32, torch.float32)
        v, r, _ = run(st, dr, dh)
        check(st, v, r, dr, dh)
    st = make(20, 264, torch.float32, torch.float32, pre=LAYER, block=False)              # the norm of the stream alone
    dr, dh = incoming(20, 264, torch.float32, torch.float32)
    v, r, _ = run(st, dr, dh)
    check(st, v, r, dr, dh)


@pytest.mark.parametrize("post,gate", [(NONE, True), (RMS, None), (LAYER, True)])
def test_without_pre_norm(post, gate):
    """No pre norm: h is None and r's gradient is the only one that arrives."""
    st = make(33, 264, torch.float32, torch.bfloat16, gate=gate, post=post, pre=NONE)
    dr, _ = incoming(33, 264, torch.float32, torch.float32)
    v, r, h = run(st, dr, None)
    assert h is None
    check(st, v, r, dr, None)


@pytest.mark.parametrize("tx,ty,th", [(torch.float32, torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16, torch.float32),
                                      (torch.float32, torch.float32, torch.bfloat16), (torch.float32, None, torch.bfloat16),
                                      (torch.bfloat16, None, torch.float32)])
def test_output_of_another_type(tx, ty, th):
    """h's gradient comes in h's type; the kernel takes it in the branch's (without one in its own, or bf16 beside a bf16 stream)."""
    st = make(21, 264, tx, ty or tx, gate=True, post=LAYER, pre=LAYER, block=ty is not None)
    dr, dh = incoming(21, 264, tx, th)
    v, r, h = run(st, dr, dh, h_dtype=th)
    assert h.dtype == th
    check(st, v, r, dr, dh.to(ty or (tx if tx == torch.bfloat16 else th)))


def test_eight_bit_outputs():
    """An 8-bit h has no gradient, and e4m3 codes are worth nothing without their scales: both belong to nq_block_norm."""
    st = make(9, 256, torch.float32, torch.float32, gate=True)
    for dtype in (torch.int8, torch.float8_e4m3fn):
        with pytest.raises(ValueError):
            fb.block_norm(leaf(st["x"]), st["y"], st["post_weight"], st["gate"], st["pre_weight"], h_dtype=dtype, h_scale=0.02)
    with pytest.raises(ValueError):
        fb.block_norm(st["x"], st["y"], st["post_weight"], st["gate"], st["pre_weight"], h_dtype=torch.float8_e4m3fn)
    r, h = fb.block_norm(st["x"], st["y"], st["post_weight"], st["gate"], st["pre_weight"], h_dtype=torch.int8, h_scale=0.02)     # no gradient wanted
    want_r, want_h, _ = nq.nq_block_norm(st["x"], st["y"], post=RMS, post_weight=st["post_weight"], gate=st["gate"], pre_weight=st["pre_weight"],
                                         h_dtype=torch.int8, h_scale=0.02)
    assert torch.equal(r, want_r) and torch.equal(h, want_h)
    x = st["x"].clone()
    with pytest.raises(TypeError):
        fb.block_norm(x, st["y"], st["post_weight"], st["gate"], st["pre_weight"], r_out=x)      # autograd would not see the write
    assert torch.equal(x, st["x"])
    dr, dh = incoming(9, 256, torch.float32, torch.float32)
    v, r, _ = run(st, dr, dh, h_scale=0.02)                        # of no meaning for an fp32 h, as in nq_block_norm
    check(st, v, r, dr, dh)


def test_second_derivatives_are_refused():
    """Gradients out of kernels are no constants: a loss that contains them must not be differentiated as if they were, whether
    or not the gradients that arrived themselves depend on the leaves."""
    x, w = torch.randn(40, 128, device="cuda").requires_grad_(True), torch.randn(64, 128, device="cuda").requires_grad_(True)
    p = torch.ones(128, device="cuda").requires_grad_(True)
    for through in (lambda y: y.square().sum(), lambda y: y.sum()):
        for wrt in (x, w):
            y = fb.fp8_linear(x, w)
            d, = torch.autograd.grad(through(y), wrt, create_graph=True)
            with pytest.raises(RuntimeError, match="differentiated again"):
                (y.sum() + d.square().sum()).backward()
        for wrt in (x, p):
            r, h = fb.block_norm(x, None, None, None, p)
            d, = torch.autograd.grad(through(h), wrt, create_graph=True)
            with pytest.raises(RuntimeError, match="differentiated again"):
                (h.sum() + d.square().sum()).backward()
    x.grad = w.grad = None
    # a graph of the gradients that is not used does no harm, and the bias's gradient is a sum that autograd knows
    b = torch.zeros(64, device="cuda").requires_grad_(True)
    fb.fp8_linear(x, w, b).square().sum().backward(create_graph=True)
    once = [t.grad.detach().clone() for t in (x, w, b)]
    x.grad = w.grad = b.grad = None
    fb.fp8_linear(x, w, b).square().sum().backward()
    assert all(torch.equal(a, t.grad) for a, t in zip(once, (x, w, b)))
    x.grad = w.grad = b.grad = None
    y = fb.fp8_linear(x, w, b)
    db, = torch.autograd.grad(y.square().sum(), b, create_graph=True)
    again, = torch.autograd.grad(db.sum(), b)
    assert torch.equal(again, torch.full_like(b, 2.0 * 40))        # d/db of sum over rows of 2 y


@pytest.mark.parametrize("options", [dict(), dict(foreach=False), dict(fused=True)], ids=["default", "each", "fused"])
def test_weights_laid_out_before_a_step_are_not_served(options):
    torch.manual_seed(6)
    stack = fb.MlpStack(2, 128, 256)
    x = torch.randn(65, 128, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(RuntimeError):
        stack.serve(x)                                             # never laid out
    stack.freeze()
    before = stack.serve(x)
    assert torch.equal(before, stack.serve(x))
    optimiser = torch.optim.AdamW(stack.parameters(), lr=0.1, **options)
    loss = stack(x).float().square().mean()
    assert torch.equal(before, stack.serve(x))                     # a forward pass alone changes nothing
    loss.backward()
    optimiser.step()
    with pytest.raises(RuntimeError):
        stack.serve(x)
    stack.freeze()
    fresh = fb.MlpStack(2, 128, 256)
    fresh.load_state_dict(stack.state_dict())
    fresh.freeze()
    assert torch.equal(stack.serve(x), fresh.serve(x)) and not torch.equal(before, stack.serve(x))
    fresh.load_state_dict(fb.MlpStack(2, 128, 256).state_dict())
    with pytest.raises(RuntimeError):
        fresh.serve(x)
    fresh.freeze()
    for p in fresh.parameters():
        p.requires_grad_(False)
    v = x.clone().requires_grad_(True)
    fresh(v).float().sum().backward()                              # through weights that are not trained
    fresh.serve(x)
    fresh.blocks[1].down = torch.nn.Parameter(fresh.blocks[1].down.detach().clone())
    with pytest.raises(RuntimeError):
        fresh.serve(x)


def test_copies_of_a_laid_out_stack(tmp_path):
    torch.manual_seed(7)
    stack = fb.MlpStack(1, 128, 256)
    x = torch.randn(9, 128, device="cuda", dtype=torch.bfloat16)
    stack.freeze()
    want = stack.serve(x)
    torch.save(stack, tmp_path / "stack")
    for twin in (copy.deepcopy(stack), torch.load(tmp_path / "stack", weights_only=False)):
        assert torch.equal(twin.serve(x), want)
        with torch.no_grad():
            twin.blocks[0].up.mul_(2.0)
        with pytest.raises(RuntimeError):
            twin.serve(x)
        with pytest.raises(RuntimeError):
            copy.deepcopy(twin).serve(x)
    state = stack.blocks[0].__getstate__()
    del state["_served_from"]                                      # a block that was stored without it
    stored = fb.MlpBlock.__new__(fb.MlpBlock)
    stored.__setstate__(state)
    with pytest.raises(RuntimeError):
        stored.serve(torch.zeros(1, 128, device="cuda").to(torch.float8_e4m3fn), torch.ones(1, 1, device="cuda"))
    assert torch.equal(stack.serve(x), want)
    with torch.inference_mode():
        assert torch.equal(stack.serve(x), want)
