"""The block-scaled e4m3 product against the definition in 64 bits: one row to many, ragged sizes, both scale layouts, output
types, pitches and alignments, bias, accumulation, the three products of a linear layer, NaN, refusals.

Tolerances.  Products of two e4m3 numbers are exact in fp32.  A group's 128 of them are added in the tensor core, where
each addition may cut at 2^-23 of what has been added: 128 * 2^-23 = 2^-16 of the group's sum of magnitudes.  The groups
are added in fp32, three roundings each: 3 G * 2^-24 for G groups.  bf16 output: another 2^-8 of itself.  Operands that
are small integers with scales that are powers of two give sums that fp32 holds exactly: those have to be equal."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from fp8_reference import spread

pytestmark = pytest.mark.gpu


def pitched(t, extra=0):
    rows, cols = t.shape
    buf = torch.full((rows, -(-cols // 16) * 16 + extra), 0x7f, dtype=torch.uint8, device="cuda")      # NaN between the rows
    buf[:, :cols] = t.to(torch.float8_e4m3fn).view(torch.uint8)
    return buf.view(torch.float8_e4m3fn)[:, :cols]


def operands(M, N, K, block, seed=0, exact=True, extra=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + M * 10007 + N * 101 + K)
    G = -(-K // 128)
    rnd = lambda *s: torch.rand(*s, generator=g, device="cuda")
    if exact:
        a, b = torch.floor(rnd(M, K) * 5) - 2, torch.floor(rnd(N, K) * 5) - 2
        sa = 2.0 ** (torch.floor(rnd(G, M) * 3) - 1)
        sb = 2.0 ** (torch.floor(rnd(G, -(-N // block)) * 3) - 1)
    else:
        a = (torch.randn(M, K, generator=g, device="cuda") * 60).clamp(-448, 448)
        b = (torch.randn(N, K, generator=g, device="cuda") * 60).clamp(-448, 448)
        sa, sb = 0.01 + rnd(G, M) * 0.05, 0.001 + rnd(G, -(-N // block)) * 0.005
    return pitched(a, extra), sa, pitched(b, extra), sb


def definition(a, sa, b, sb, block):
    A = a.double() * spread(sa, 1, *a.shape).to(a.device)
    B = b.double() * spread(sb, block, *b.shape).to(b.device)
    return A @ B.t(), A.abs() @ B.abs().t()


def check(got, want, size, groups):
    tol = (2.0 ** -16 + 3 * groups * 2.0 ** -24) * size + (2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0) * want.abs()
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-300)).max())


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 4096, 4096), (1, 127, 1000), (2, 129, 129), (7, 500, 16), (15, 64, 2048), (16, 256, 384),
          (17, 300, 513), (33, 1000, 768), (37, 2048, 4096), (64, 128, 100), (65, 640, 640), (127, 127, 127), (128, 128, 128), (129, 130, 257),
          (200, 2304, 768), (300, 16, 1024), (513, 257, 300), (1000, 1100, 640), (2500, 768, 768), (2049, 2305, 1153), (300, 5000, 512),
          (4096, 4096, 256)]


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_exact_sums(M, N, K, block):
    a, sa, b, sb = operands(M, N, K, block)
    want, size = definition(a, sa, b, sb, block)
    assert float(size.max()) * 16 < 2 ** 24
    y = nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block, y_dtype=torch.float32)
    assert torch.equal(y.double(), want)
    y = nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block)
    assert torch.equal(y, want.float().to(torch.bfloat16))
    nq.nq_device_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (5, 1000, 1000), (40, 256, 700), (100, 129, 20000), (700, 900, 1024), (2100, 2400, 1300)])
def test_general_values(M, N, K, block, dtype):
    a, sa, b, sb = operands(M, N, K, block, exact=False)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(3)).cuda()
    want, size = definition(a, sa, b, sb, block)
    got = nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block, bias=bias, y_dtype=dtype)
    check(got, want + bias.double(), size + bias.abs().double(), -(-K // 128))
    assert torch.equal(got, nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=block, bias=bias, y_dtype=dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pitch,offset", [(1040, 0), (1000, 0), (1001, 0), (1008, 1), (1004, 4)])
@pytest.mark.parametrize("M", [3, 150, 2000])
def test_output_pitch_and_alignment(M, pitch, offset, dtype):
    N, K = 1000, 640
    a, sa, b, sb = operands(M, N, K, 128, extra=32)
    want, _ = definition(a, sa, b, sb, 128)
    buf = torch.full((M * pitch + offset + 8,), 7.0, dtype=dtype, device="cuda")
    y = buf[offset:offset + M * pitch].view(M, pitch)[:, :N]
    assert nq.nq_fp8_gemm(a, sa, b, sb, y_out=y) is y
    assert torch.equal(y, want.float().to(dtype))
    rest = buf.clone()
    rest[offset:offset + M * pitch].view(M, pitch)[:, :N] = 7.0
    assert bool((rest == 7.0).all())                                       # nothing beside the matrix is written


@pytest.mark.parametrize("M,N,K", [(1, 200, 512), (70, 300, 300), (2000, 1024, 384), (2000, 1025, 384)])
def test_accumulate_and_bias(M, N, K):
    a, sa, b, sb = operands(M, N, K, 1)
    want, _ = definition(a, sa, b, sb, 1)
    bias = torch.floor(torch.rand(N, device="cuda") * 9) - 4
    y = torch.floor(torch.rand(M, N, device="cuda") * 100)
    old = y.double()
    nq.nq_fp8_gemm(a, sa, b, sb, b_block_rows=1, bias=bias, y_out=y, accumulate=True)
    assert torch.equal(y.double(), want + bias.double() + old)


def test_scale_pitch_and_views():
    """Scales and operands that are parts of larger tensors."""
    M, N, K = 70, 260, 512
    a, sa, b, sb = operands(M, N, K, 128, extra=64)
    want, _ = definition(a, sa, b, sb, 128)
    big = torch.zeros(4, M + 5, device="cuda")
    big[:, 2:2 + M] = sa
    y = nq.nq_fp8_gemm(a, big[:, 2:2 + M], b, sb, y_dtype=torch.float32)
    assert torch.equal(y.double(), want)
    y = nq.nq_fp8_gemm(a[:, 128:], sa[1:], b[:, 128:], sb[1:], y_dtype=torch.float32)     # without the first group
    w2, _ = definition(a[:, 128:], sa[1:], b[:, 128:], sb[1:], 128)
    assert torch.equal(y.double(), w2)


@pytest.mark.parametrize("tokens,d_in,d_out", [(5, 256, 384), (130, 200, 300), (1500, 768, 1100)])
def test_linear_layer_and_its_gradients(tokens, d_in, d_out):
    """x W^T, dy W and dy^T x through the quantiser, against 64-bit products of what the codes stand for, and against
    differences of the loss <dy, x W^T> of those values."""
    g = torch.Generator().manual_seed(tokens)
    x, w, dy = (torch.randn(*s, generator=g).cuda() for s in ((tokens, d_in), (d_out, d_in), (tokens, d_out)))
    qx, sx, xt, sxt = nq.nq_fp8_quantize(x.bfloat16(), transposed=True)
    qw, sw, wt, swt = nq.nq_fp8_quantize(w, block_rows=128, transposed=True)
    qd, sd, dt, sdt = nq.nq_fp8_quantize(dy.bfloat16(), transposed=True)
    for out, (a, sa, b, sb, block) in ((nq.nq_fp8_gemm(qx, sx, qw, sw, y_dtype=torch.float32), (qx, sx, qw, sw, 128)),
                                       (nq.nq_fp8_gemm(qd, sd, wt, swt, y_dtype=torch.float32), (qd, sd, wt, swt, 128)),
                                       (nq.nq_fp8_gemm(dt, sdt, xt, sxt, b_block_rows=1, y_dtype=torch.float32), (dt, sdt, xt, sxt, 1))):
        want, size = definition(a, sa, b, sb, block)
        check(out, want, size, -(-a.shape[1] // 128))
    # differences: the loss is linear in each factor, so a step of 1 is as good as any
    W = qw.double() * spread(sw, 128, *qw.shape).cuda()
    D = qd.double() * spread(sd, 1, *qd.shape).cuda()
    X = x.double()
    way = torch.randn(tokens, d_in, generator=g).cuda().double()
    loss = lambda v: (D * (v @ W.t())).sum()
    diff = (loss(X + way) - loss(X - way)) / 2
    dx = nq.nq_fp8_gemm(qd, sd, wt, swt, y_dtype=torch.float32).double()
    size = (D.abs() @ W.abs() * way.abs()).sum()
    assert abs(float((dx * way).sum() - diff)) <= (2.0 ** -16 + 3 * 9 * 2.0 ** -24) * float(size)


def test_nan_stays_where_it_belongs():
    M, N, K = 140, 300, 512
    a, sa, b, sb = operands(M, N, K, 128)
    sa[2, 5] = float("nan")
    sb[1, 2] = float("inf")
    y = nq.nq_fp8_gemm(a, sa, b, sb, y_dtype=torch.float32)
    bad = ~torch.isfinite(y)
    assert bool(bad[5].all()) and bool(bad[:, 256:].all())
    bad[5] = False
    assert not bool(bad[:, :256].any())


def test_empty():
    for M, N, K in ((0, 64, 128), (64, 0, 128)):
        a, sa, b, sb = (torch.empty(s, device="cuda") for s in ((M, K), (1, M), (N, K), (1, N)))
        assert nq.nq_fp8_gemm(a.to(torch.float8_e4m3fn), sa, b.to(torch.float8_e4m3fn), sb, b_block_rows=1).shape == (M, N)
    a, b = torch.empty(3, 0, device="cuda").to(torch.float8_e4m3fn), torch.empty(40, 0, device="cuda").to(torch.float8_e4m3fn)
    bias = torch.randn(40, device="cuda")
    y = nq.nq_fp8_gemm(a, torch.empty(0, 3, device="cuda"), b, torch.empty(0, 1, device="cuda"), bias=bias, y_dtype=torch.float32)
    assert torch.equal(y, bias.expand(3, 40))


def test_other_stream():
    a, sa, b, sb = operands(300, 400, 512, 128)
    want, _ = definition(a, sa, b, sb, 128)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = nq.nq_fp8_gemm(a, sa * 2, b, sb, y_dtype=torch.float32)
    side.synchronize()
    assert torch.equal(y.double(), 2 * want)


def test_refusals():
    a, sa, b, sb = operands(32, 64, 256, 128)
    for k in [dict(a=a.float()), dict(b=b.view(torch.uint8)), dict(a=a[:, :128]), dict(sa=sa[:1]), dict(sb=sa), dict(sa=sa.double()),
              dict(b_block_rows=2), dict(b_block_rows=1), dict(bias=torch.zeros(32, device="cuda")), dict(y_out=torch.zeros(32, 65, device="cuda")),
              dict(y_out=torch.zeros(64, 32, device="cuda").t()), dict(accumulate=True), dict(y_dtype=torch.float16), dict(a=a.cpu()),
              dict(sa=sa.t().contiguous().t())]:
        with pytest.raises(ValueError):
            nq.nq_fp8_gemm(**{**dict(a=a, sa=sa, b=b, sb=sb), **k})
    for k in [dict(a=a[:, 8:], b=b[:, 8:], sa=sa, sb=sb),                             # starts off 16 bytes
              dict(y_out=torch.zeros(32, 64, device="cuda", dtype=torch.bfloat16), accumulate=True),
              dict(a=torch.zeros(32 * 264, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).view(32, 264)[:, :256])]:   # pitch
        with pytest.raises(nq.NqError):
            nq.nq_fp8_gemm(**{**dict(a=a, sa=sa, b=b, sb=sb), **k})
