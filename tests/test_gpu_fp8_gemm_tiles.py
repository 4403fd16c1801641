"""The block-scaled product where a thread block works through many tiles with little to do in each: ragged last tiles, whose
warps partly lie outside the matrix, between whole ones, with one or two groups of K.

Operands are small integers with scales that are powers of two, and so is the bias: every sum is exact in fp32, so results
have to be equal."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from test_gpu_fp8_gemm import definition, operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("M,N,K", [(2100, 24000, 128), (2100, 23900, 64), (260, 40000, 100), (4390, 12345, 256)])
def test_bias_of_each_tile(M, N, K, block):
    """A warp without rows (M % 256 below 224) or columns (N % 256 below 129) of its own must leave nothing behind that reaches
    its next tile's bias: neighbouring tiles' biases differ everywhere."""
    a, sa, b, sb = operands(M, N, K, block)
    want, _ = definition(a, sa, b, sb, block)
    bias = (torch.arange(N, device="cuda") * 37 % 1009).float() - 504
    want = want + bias.double()
    for _ in range(3):
        y = nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block, bias=bias, y_dtype=torch.float32)
        assert torch.equal(y.double(), want)
    y = nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block, bias=bias)
    assert torch.equal(y, want.float().to(torch.bfloat16))
    nq.nq_device_status()


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("bias", [False, True])
def test_scales_that_are_no_numbers(block, bias):
    """A NaN or infinite scale shows in its row, or in the columns of its block, and nowhere else."""
    M, N, K = 2000, 2304, 640
    a, sa, b, sb = operands(M, N, K, block)
    want, _ = definition(a, sa, b, sb, block)
    add = (torch.arange(N, device="cuda") % 17).float() if bias else None
    want = want if add is None else want + add.double()
    sa[2, 1500], sa[0, 127], sa[4, 1999] = float("nan"), float("inf"), float("nan")
    at = 2 if block == 128 else 300
    sb[1, at], sb[3, -1] = float("inf"), float("nan")
    columns = torch.zeros(N, dtype=torch.bool, device="cuda")
    columns[at * block:(at + 1) * block] = True
    columns[(sb.shape[1] - 1) * block:] = True
    rows = torch.zeros(M, dtype=torch.bool, device="cuda")
    rows[[127, 1500, 1999]] = True
    for dtype in (torch.float32, torch.bfloat16):
        y = nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block, bias=add, y_dtype=dtype)
        assert torch.equal(~torch.isfinite(y), rows[:, None] | columns[None, :])
        good = (~rows[:, None] & ~columns[None, :])
        assert torch.equal(y[good], want.float().to(dtype)[good])
    nq.nq_device_status()
