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
