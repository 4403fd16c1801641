"""The block norm's 8-bit outputs where thread blocks work through many rows, and rows alone against the same rows among many.

An fp32 h is the value that the 8-bit outputs are rounded from, so the quantiser's codes and scales of it have to be those of the
e4m3 output, and its nearest whole numbers those of the INT8 output, bit for bit; test_gpu_block_norm.py holds h to the
definition.  A row's sums are added in one order however many rows there are: alone or among others it has the same bits."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from test_gpu_block_norm import LAYER, NONE, RMS, check, make, split
from test_gpu_fp8_gemm import check as check_product, definition

pytestmark = pytest.mark.gpu

# rows enough for two and more to each thread block of a full machine (148 SMs x the blocks that fit), by width
CASES = [(9001, 264, 0), (4801, 512, 0), (4801, 768, 197), (2501, 1138, 0), (2501, 1144, 1), (1301, 4096, 50), (1301, 4097, 0), (701, 8192, 0),
         (701, 8191, 300), (601, 9000, 0), (601, 9001, 0), (3001, 200, 0)]


def placed(t, pitch, offset):
    rows, cols = t.shape
    buf = torch.full((rows * pitch + offset,), 1e3, dtype=t.dtype, device="cuda")
    v = buf[offset:].view(rows, pitch)[:, :cols]
    v.copy_(t)
    return v


@pytest.mark.parametrize("tx,ty", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("rows,cols,group", CASES)
def test_eight_bit_outputs_of_many_rows(rows, cols, group, kind, tx, ty):
    st = make(rows, cols, tx, ty, gate=True, group=group, post=kind, pre=kind, bias=kind == LAYER)
    if cols == 1144:                                               # whole pieces, rows that start anywhere
        st["x"], st["y"] = placed(st["x"], 1147, 1), placed(st["y"], 1145, 3)
    if cols == 512:                                                # no post norm
        st["post"], st["post_weight"], st["post_bias"] = NONE, None, None
    _, h = check(st, h_dtype=torch.float32)
    x, y, how = split(st)
    q, s, _, _ = nq.nq_fp8_quantize(h)
    _, h8, hs = nq.nq_block_norm(x, y, h_dtype=torch.float8_e4m3fn, **how)
    assert torch.equal(hs, s)
    assert torch.equal(h8.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8))
    _, hi, none = nq.nq_block_norm(x, y, h_dtype=torch.int8, h_scale=0.02, **how)
    inv = torch.tensor(1.0, device="cuda") / torch.tensor(0.02, device="cuda")
    assert none is None and torch.equal(hi, torch.clamp(torch.round(h * inv), -128, 127).to(torch.int8))
    nq.nq_device_status()


def test_rows_alone_and_among_many():
    """What a token's serving goes through, step by step: norm to e4m3, product, quantiser."""
    for rows, cols, hidden in ((3000, 768, 1536), (1500, 4096, 1000), (2000, 1138, 900)):
        st = make(rows, cols, torch.bfloat16, torch.bfloat16, gate=True)
        g = torch.Generator(device="cuda").manual_seed(cols)
        w, sw, _, _ = nq.nq_fp8_quantize(torch.randn(hidden, cols, generator=g, device="cuda") * cols ** -0.5, block_rows=128)
        x, y, how = split(st)
        r, h, hs = nq.nq_block_norm(x, y, h_dtype=torch.float8_e4m3fn, **how)
        z = nq.nq_fp8_gemm(h, hs, w, sw)
        q, s, _, _ = nq.nq_fp8_quantize(z)
        for few in (1, 3, 40):
            r1, h1, hs1 = nq.nq_block_norm(x[:few], y[:few], h_dtype=torch.float8_e4m3fn, **how)
            assert torch.equal(r1, r[:few]) and torch.equal(hs1, hs[:, :few])
            assert torch.equal(h1.contiguous().view(torch.uint8), h[:few].contiguous().view(torch.uint8))
            q1, s1, _, _ = nq.nq_fp8_quantize(z[:few])
            assert torch.equal(s1, s[:, :few]) and torch.equal(q1.contiguous().view(torch.uint8), q[:few].contiguous().view(torch.uint8))
            want, size = definition(h1, hs1, w, sw, 128)          # split over K in another way, so within the product's bound, each of them
            groups = -(-cols // 128)
            check_product(nq.nq_fp8_gemm(h1, hs1, w, sw), want, size, groups)
            check_product(z[:few], want, size, groups)
