"""Tensors of more than 2^31 elements: the last rows are computed at the right places by all e4m3 and block-norm kernels."""
import numpy as np
import pytest
import torch

import paper_2506_17870_b200 as nq
from fp8_reference import quantize

pytestmark = pytest.mark.gpu


def filled(rows, cols, dtype, tail):
    """Zeros with `tail` in the last rows."""
    t = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    t[-len(tail):] = tail
    return t


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def test_quantiser():
    rows, cols = 70000, 32768                                       # 2.29e9 elements
    tail = torch.randn(128 + rows % 128, cols, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    q, s, qt, st = nq.nq_fp8_quantize(filled(rows, cols, torch.bfloat16, tail.cuda()), transposed=True)
    want_q, want_s = quantize(tail.float().numpy(), 1)
    n = len(tail)
    assert np.array_equal(q[-n:].float().cpu().numpy(), want_q) and np.array_equal(s[:, -n:].cpu().numpy(), want_s)
    last = tail[-(rows % 128):].float().numpy()                     # the last, short group of the transpose
    want_q, want_s = quantize(np.ascontiguousarray(last.T), 1)
    assert np.array_equal(qt[:, -(rows % 128):].float().cpu().numpy(), want_q) and np.array_equal(st[-1:].cpu().numpy(), want_s)


@pytest.mark.parametrize("M,N,K", [(600000, 4096, 256), (4200000, 640, 520), (9000000, 256, 128)])
def test_product(M, N, K):
    """2.3e9 to 2.7e9 outputs, and an operand of 2.2e9; small integers, so the sums are exact."""
    g = torch.Generator(device="cuda").manual_seed(2)
    pitch = -(-K // 16) * 16
    a = torch.zeros((M, pitch), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :K]
    tail = torch.floor(torch.rand(300, K, generator=g, device="cuda") * 5) - 2
    a[-300:].view(torch.uint8).copy_(tail.to(torch.float8_e4m3fn).view(torch.uint8))
    b = (torch.floor(torch.rand(N, pitch, generator=g, device="cuda") * 5) - 2).to(torch.float8_e4m3fn)[:, :K]
    sa = torch.ones(-(-K // 128), M, device="cuda")
    sa[:, -300:] = 2.0
    sb = torch.full((-(-K // 128), -(-N // 128)), 0.5, device="cuda")
    y = nq.nq_fp8_gemm(a, sa, b, sb)
    want = tail.double() @ b.double().t()
    assert torch.equal(y[-300:], want.to(torch.bfloat16))
    assert bool((y[-1300:-300] == 0).all()) and bool((y[:1000] == 0).all())
    nq.nq_device_status()


def test_block_norm_and_its_backward():
    rows, cols = 140000, 16384                                      # 2.29e9 elements
    n = 200
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda: torch.randn(n, cols, generator=g, device="cuda").to(torch.bfloat16)
    tx, ty, td = rnd(), rnd(), rnd()
    w = 1 + 0.1 * torch.randn(cols, generator=g, device="cuda")
    how = dict(post=nq.NQ_NORM_RMS, post_weight=w, pre=nq.NQ_NORM_RMS, pre_weight=w)
    x, y = filled(rows, cols, torch.bfloat16, tx), filled(rows, cols, torch.bfloat16, ty)
    r, h, _ = nq.nq_block_norm(x, y, **how)
    small_r, small_h, _ = nq.nq_block_norm(tx, ty, **how)
    assert torch.equal(r[-n:], small_r) and torch.equal(h[-n:], small_h)
    assert bool((h[:1000] == 0).all())
    del h
    d = filled(rows, cols, torch.bfloat16, td)
    got = nq.nq_block_norm_backward(r, y, dr=d, dh=d, **how)
    small = nq.nq_block_norm_backward(small_r, ty, dr=td, dh=td, **how)
    assert torch.equal(got[0][-n:], small[0]) and torch.equal(got[1][-n:], small[1])
    for a, b in ((got[3], small[3]), (got[5], small[5])):           # sums over rows of which all others are zero
        assert float((a - b).abs().max()) <= 2.0 ** -16 * float(b.abs().max()) * 8
    nq.nq_device_status()
