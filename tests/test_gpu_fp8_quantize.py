"""The e4m3 quantiser: bit for bit against its definition, matrix and transpose, ragged sizes, pitches and alignments,
zeros, tiny values, infinities and NaN; its refusals."""
import numpy as np
import pytest
import torch

import paper_2506_17870_b200 as nq
from fp8_reference import quantize, round_e4m3

pytestmark = pytest.mark.gpu


def values(rows, cols, dtype, seed=0):
    rng = np.random.default_rng(1000 * rows + cols + seed)
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=(1, cols)))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def same(q, s, ref):
    want_q, want_s = ref
    got = q.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(s.cpu().numpy().view(np.uint32) & 0x7fffffff, want_s.view(np.uint32) & 0x7fffffff) or \
        np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)
    assert np.array_equal(got, want_q, equal_nan=True)


def check(x, block_rows, rowwise=True, transposed=True):
    f = x.float().cpu().numpy()
    q, s, qt, st = nq.nq_fp8_quantize(x, block_rows=block_rows, rowwise=rowwise, transposed=transposed)
    assert (q is None) == (not rowwise) and (qt is None) == (not transposed)
    if rowwise:
        assert q.stride(0) % 16 == 0 or q.shape[0] == 1
        same(q, s, quantize(f, block_rows))
    if transposed:
        same(qt, st, quantize(np.ascontiguousarray(f.T), block_rows))


SIZES = [(1, 1), (1, 128), (1, 4096), (3, 127), (5, 129), (127, 16), (128, 128), (129, 257), (130, 384), (200, 1000), (385, 640), (1000, 100)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, block_rows, dtype):
    check(values(rows, cols, dtype).cuda(), block_rows)


@pytest.mark.parametrize("rowwise,transposed", [(True, False), (False, True)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_one_side_only(block_rows, rowwise, transposed):
    check(values(150, 300, torch.bfloat16).cuda(), block_rows, rowwise, transposed)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pitch,offset", [(320, 0), (320, 16), (304, 8), (301, 0), (303, 1), (257, 3)])
def test_pitch_and_alignment(pitch, offset, dtype):
    rows, cols = 140, 250
    buf = torch.full((rows * pitch + offset + 16,), 1e4, dtype=dtype, device="cuda")     # what lies between rows is large
    x = buf[offset:offset + rows * pitch].view(rows, pitch)[:, :cols]
    x.copy_(values(rows, cols, dtype))
    check(x, 1)
    check(x, 128)


def test_padding_is_not_written():
    rows, cols, pitch = 37, 100, 160
    x = values(rows, cols, torch.float32).cuda()
    q = torch.full((rows, pitch), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.empty((1, rows), device="cuda")
    qt = torch.full((cols, 96), 0x55, dtype=torch.uint8, device="cuda")
    st = torch.empty((1, cols), device="cuda")
    L = nq.lib()
    assert L.nq_fp8_quantize(x.data_ptr(), cols, nq.NQ_F32, rows, cols, 1, q.data_ptr(), pitch, s.data_ptr(), rows, qt.data_ptr(), 96,
                             st.data_ptr(), cols, torch.cuda.current_stream().cuda_stream) == 0
    assert bool((q[:, cols:] == 0x55).all()) and bool((qt[:, rows:] == 0x55).all())
    same(q.view(torch.float8_e4m3fn)[:, :cols], s, quantize(x.cpu().numpy(), 1))


@pytest.mark.parametrize("block_rows", [1, 128])
def test_special_values(block_rows):
    x = values(260, 260, torch.float32)
    x[0, :128] = 0.0                                     # a group of zeros
    x[1, :128] = 1e-42                                   # subnormal: the scale stays a normal number
    x[2, :128] = 3.3e38
    x[131, 140] = float("nan")
    x[132, 3] = float("inf")
    x[133, 4] = -float("inf")
    x[200] = torch.arange(260) / 16.0                    # ties of the rounding
    check(x.cuda(), block_rows)


def test_all_codes_round_to_themselves():
    from fp8_reference import E4M3
    x = torch.zeros(2, 128)
    x[0, :127] = torch.from_numpy(E4M3).float()
    x[1, :126] = torch.from_numpy((E4M3[:-1] + E4M3[1:]) / 2).float()      # midpoints: to the even code
    x[1, 127] = 448.0
    q, s, _, _ = nq.nq_fp8_quantize(x.cuda())
    assert s.flatten().tolist() == [1.0, 1.0]
    assert torch.equal(q.float().cpu()[0, :127], x[0, :127])
    assert np.array_equal(q.float().cpu().numpy()[1], round_e4m3(x[1].double().numpy()))


def test_other_stream():
    x = values(300, 500, torch.bfloat16).cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = x * 2
        q, s, _, _ = nq.nq_fp8_quantize(y)
    side.synchronize()
    same(q, s, quantize(y.float().cpu().numpy(), 1))


def test_empty():
    for shape in ((0, 40), (40, 0)):
        q, s, qt, st = nq.nq_fp8_quantize(torch.empty(shape, device="cuda"), transposed=True)
        assert q.shape == shape and qt.shape == shape[::-1]


def test_refusals():
    x = torch.zeros(8, 32, device="cuda")
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x, block_rows=64)
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x.half())
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x.cpu())
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x.t())
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x[0])
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x[:1].expand(8, 32))
    with pytest.raises(ValueError):
        nq.nq_fp8_quantize(x, rowwise=False)
    L, q = nq.lib(), torch.zeros(8 * 48, dtype=torch.uint8, device="cuda")
    s = torch.zeros(64, device="cuda")
    P = lambda t, o=0: t.data_ptr() + o
    args = lambda **k: [{**dict(x=P(x), ldx=32, t=0, rows=8, cols=32, b=1, q=P(q), ldq=32, s=P(s), lds=8, qt=None, ldqt=0, st=None, ldst=0, z=None), **k}[n]
                        for n in ("x", "ldx", "t", "rows", "cols", "b", "q", "ldq", "s", "lds", "qt", "ldqt", "st", "ldst", "z")]
    for want, change in ((1, dict(rows=-1)), (1, dict(ldx=31)), (1, dict(t=2)), (1, dict(b=2)), (1, dict(q=None)), (1, dict(s=None)),
                         (1, dict(q=None, s=None)), (1, dict(lds=7)), (1, dict(ldq=16)), (1, dict(qt=P(q))), (3, dict(ldq=40)),
                         (3, dict(q=P(q, 8))), (3, dict(x=P(x, 2))), (3, dict(s=P(s, 2))), (2, dict(rows=1 << 31)), (1, dict(x=None))):
        assert L.nq_fp8_quantize(*args(**change)) == want, change
