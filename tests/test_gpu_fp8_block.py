"""The e4m3 stack end to end: autograd wiring against the entry points, gradients against the same stack in 64 bits, serving
against training, the INT8 hand-over against the oracle's product.

Tolerances.  Rounding to e4m3 costs a value 2.6 % in the root mean square (half a step of 2^-3 .. 2^-4, evenly spread), so a
product of two rounded matrices with random signs is off by about 3.7 % of its norm, and a chain of n products adds up
to about 3.7 % * sqrt(n).  A stack of two blocks has 4 products forward and at most 4 more on a gradient's way: 11 %; twice
that is allowed."""
import numpy as np
import pytest
import torch

import oracle
import paper_2506_17870_b200 as nq
from fp8_reference import norm
from paper_2506_17870_b200 import fp8_block as fb
from paper_2506_17870_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def test_linear_is_its_three_products():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(300, 256, generator=g).cuda().bfloat16().requires_grad_(True)
    w = torch.randn(384, 256, generator=g).cuda().requires_grad_(True)
    b = torch.randn(384, generator=g).cuda().requires_grad_(True)
    dy = torch.randn(300, 384, generator=g).cuda().bfloat16()
    y = fb.fp8_linear(x, w, b)
    y.backward(dy)
    qx, sx, xt, sxt = nq.nq_fp8_quantize(x.detach(), transposed=True)
    qw, sw, wt, swt = nq.nq_fp8_quantize(w.detach(), block_rows=128, transposed=True)
    qd, sd, dt, sdt = nq.nq_fp8_quantize(dy, transposed=True)
    assert torch.equal(y, nq.nq_fp8_gemm(qx, sx, qw, sw, bias=b.detach()))
    assert torch.equal(x.grad, nq.nq_fp8_gemm(qd, sd, wt, swt))
    assert torch.equal(w.grad, nq.nq_fp8_gemm(dt, sdt, xt, sxt, b_block_rows=1, y_dtype=torch.float32))
    assert torch.equal(b.grad, dy.float().sum(0))


def in_64_bits(stack, x, params):
    y = None
    n = len(stack.blocks)
    for i in range(n + 1):
        pre = params[f"blocks.{i}.pre_weight"] if i < n else params["final_weight"]
        if y is not None:
            u = norm(y, 1, params[f"blocks.{i - 1}.post_weight"], None, 1e-6) * params[f"blocks.{i - 1}.gate"]
            x = stack.how["skip_scale"] * x + stack.how["branch_scale"] * u
        h = norm(x, 1, pre, None, 1e-6)
        if i < n:
            p = lambda k: params[f"blocks.{i}.{k}"]
            y = torch.nn.functional.gelu(h @ p("up").t() + p("up_bias")) @ p("down").t()
    return h


def test_stack_gradients():
    torch.manual_seed(3)
    stack = fb.MlpStack(2, 256, 640, skip_scale=0.8, branch_scale=1.1)
    x = torch.randn(500, 256, device="cuda", dtype=torch.bfloat16)
    dh = torch.randn(500, 256, device="cuda", dtype=torch.bfloat16)
    stack(x).backward(dh)
    params = {k: v.detach().double().requires_grad_(True) for k, v in stack.named_parameters()}
    want = in_64_bits(stack, x.double(), params)
    (want * dh.double()).sum().backward()
    far = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())
    with torch.no_grad():
        assert far(stack(x), want) < 0.22
    for name, p in stack.named_parameters():
        assert far(p.grad, params[name].grad) < 0.22, name


def test_served_as_trained():
    torch.manual_seed(4)
    stack = fb.MlpStack(2, 384, 768)
    x = torch.randn(257, 384, device="cuda", dtype=torch.bfloat16)
    with torch.no_grad():
        trained = stack(x).float()
    stack.freeze()
    many = stack.serve(x).float()
    assert float((many - trained).norm() / trained.norm()) < 0.22
    for rows in (1, 3, 40):                                        # a token's result does not depend on its batch beyond rounding
        some = stack.serve(x[:rows]).float()
        assert float((some - many[:rows]).norm() / some.norm()) < 0.22


def test_training_lowers_the_loss():
    losses = fb.main(steps=25, tokens=512, width=256, hidden=512, blocks=2)
    assert losses[-1] < 0.7 * losses[0]


@pytest.mark.parametrize("part", [False, True])
def test_int8_hand_over(part):
    """Layer norm to INT8 ahead of a nested linear: the product's accumulators are the oracle's on the norm's INT8 output."""
    rows, cols, out, h_bits, act = 33, 768, 200, 5, 0.03
    d = wl.gemm_inputs(77, 1, rows, out, cols)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    lin = fb.NestedLinear(dev(d["W"]), dev(d["w_scale"]), h_bits, act, dev(d["mask"]))
    g = torch.Generator().manual_seed(5)
    x, w, b = torch.randn(rows, cols, generator=g).cuda(), torch.rand(cols, generator=g).cuda() + 0.5, torch.randn(cols, generator=g).cuda()
    got = lin(x, w, b, part_bit=part).cpu().numpy()
    _, h, _ = nq.nq_block_norm(x, None, pre=nq.NQ_NORM_LAYER, pre_weight=w, pre_bias=b, h_dtype=torch.int8, h_scale=act)
    wh, wlo = oracle.decompose(d["W"], d["mask"], 8, h_bits, True)
    acc = oracle.gemm_acc(h.cpu().numpy(), wh if part else d["W"])
    want = oracle.dequant(acc, d["w_scale"], act, 8 - h_bits if part else 0)
    assert np.array_equal(got, want)
