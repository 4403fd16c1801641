"""The e4m3 entry points captured into a CUDA graph: launches with programmatic dependency keep their order when they are
replayed.  Every result has to be bit for bit that of the same calls made directly."""
import pytest
import torch

import paper_2506_17870_b200 as nq

pytestmark = pytest.mark.gpu


def layer(x, y, w, gate, up, dh):
    """norm -> product -> quantised both ways -> the gradients' products -> norm backward, each on the one before."""
    how = dict(post=nq.NQ_NORM_LAYER, gate=gate, pre=nq.NQ_NORM_RMS, pre_weight=w)
    r, h, hs = nq.nq_block_norm(x, y, h_dtype=torch.float8_e4m3fn, **how)
    q, s, qt, st = nq.nq_fp8_quantize(up, block_rows=128, transposed=True)
    z = nq.nq_fp8_gemm(h, hs, q, s)
    d, sd, dt, sdt = nq.nq_fp8_quantize(z, transposed=True)
    dx = nq.nq_fp8_gemm(d, sd, qt, st)
    _, plain, _ = nq.nq_block_norm(x, y, **how)
    _, _, pt, spt = nq.nq_fp8_quantize(plain, rowwise=False, transposed=True)
    dw = nq.nq_fp8_gemm(dt, sdt, pt, spt, b_block_rows=1, y_dtype=torch.float32)
    return (r, h.view(torch.uint8), hs, z, dx, dw) + nq.nq_block_norm_backward(r, y, dr=dx, dh=dh, **how)


@pytest.mark.parametrize("rows,width,hidden", [(1, 256, 384), (45, 512, 1024), (2000, 768, 1100)])
def test_replayed(rows, width, hidden):
    g = torch.Generator(device="cuda").manual_seed(rows)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    fresh = lambda: [n(rows, width).bfloat16(), n(rows, width).bfloat16(), 1 + 0.2 * n(width), 0.5 + 0.2 * n(1, width), n(hidden, width) * width ** -0.5,
                     n(rows, width).bfloat16()]
    inputs = fresh()
    layer(*inputs)                                                 # once directly: set-up that must not be captured
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer(*inputs)
    for _ in range(4):
        for t, f in zip(inputs, fresh()):
            t.copy_(f)
        graph.replay()
        want = layer(*inputs)
        for a, b in zip(got, want):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    nq.nq_device_status()
