"""Refusals of the e4m3 and block-norm entry points that need no GPU: they come before any CUDA call."""
import ctypes

import pytest

import paper_2506_17870_b200 as nq
from paper_2506_17870_b200 import build as nq_build


@pytest.fixture(scope="module")
def L():
    nq_build.build()
    return nq.lib()


def test_quantize(L):
    call = lambda rows=4, cols=4, block=1, t=0, q=None, s=None, x=None, ldx=4: L.nq_fp8_quantize(x, ldx, t, rows, cols, block, q, 16, s, 4, None, 0, None, 0, None)
    assert call(rows=-1) == 1 and call(t=2) == 1 and call(block=64) == 1
    assert call(q=16) == 1 and call() == 1                          # one of a pair, nothing to write
    assert call(rows=0) == 0 and call(cols=0) == 0
    assert call(rows=1 << 31) == 2
    assert call(x=64, q=8, s=16) == 3 and call(x=64, q=16, s=18) == 3
    assert call(x=64, q=16, s=16, ldx=3) == 1


def test_gemm(L):
    def call(M=4, N=4, K=16, a=16, lda=16, sa=16, ldsa=4, b=16, ldb=16, sb=16, ldsb=1, block=128, y=16, ldy=4, t=0, acc=0):
        return L.nq_fp8_gemm(a, lda, sa, ldsa, b, ldb, sb, ldsb, block, None, M, N, K, y, ldy, t, acc, None)
    for change in (dict(M=-1), dict(t=2), dict(block=2), dict(y=None), dict(ldy=3), dict(a=None), dict(sb=None), dict(lda=8), dict(ldsa=3),
                   dict(block=1, ldsb=3), dict(ldsb=0)):
        assert call(**change) == 1, change
    for change in (dict(a=8), dict(b=24), dict(lda=24), dict(sa=18), dict(y=18)):
        assert call(**change) == 3, change
    assert call(acc=1, t=1) == 2 and call(M=1 << 30) == 2
    assert call(M=0) == 0 and call(N=0, y=None) == 0


def desc(**k):
    base = dict(rows=4, cols=16, ldx=16, ldy=16, ldr=16, ldh=16, lddx=16, lddy=16, lddr=16, lddh=16, rows_per_gate=0, x_dtype=0, y_dtype=0,
                h_dtype=0, post=0, pre=1, skip_scale=1.0, branch_scale=1.0, eps=1e-6, h_scale=1.0)
    return nq.nq_block_norm_desc(**{**base, **k})


def test_block_norm(L):
    def call(x=64, y=None, pw=None, pb=None, gate=None, qw=None, qb=None, r=None, h=64, hs=None, ldhs=4, **k):
        d = desc(**k)
        return L.nq_block_norm(ctypes.addressof(d), x, y, pw, pb, gate, qw, qb, r, h, hs, ldhs, None)
    for change in (dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(post=3), dict(x_dtype=1), dict(x_dtype=2), dict(h_dtype=4), dict(gate=64),
                   dict(post=1), dict(y=64, pw=64), dict(pre=0), dict(pre=0, h=None), dict(x=None), dict(h=None), dict(h_dtype=2), dict(h_dtype=2, hs=64, ldhs=3),
                   dict(h_dtype=3, h_scale=0.0), dict(ldx=15), dict(ldh=15)):
        assert call(**change) == 1, change
    assert L.nq_block_norm(None, 64, None, None, None, None, None, None, None, 64, None, 0, None) == 1
    for change in (dict(x=66), dict(h_dtype=3, h=72), dict(h_dtype=3, ldh=24), dict(qw=66), dict(h_dtype=2, hs=66)):
        assert call(**change) == 3, change
    assert call(cols=16385, ldx=16385, ldh=16385) == 2
    assert call(rows=0) == 0


def test_block_norm_backward(L):
    def call(r=64, y=None, dr=None, dh=64, pw=None, pb=None, gate=None, qw=None, dx=64, dy=None, dgate=None, dpw=None, dpb=None, dqw=None, dqb=None,
             ws=None, n=0, **k):
        d = desc(**k)
        return L.nq_block_norm_backward(ctypes.addressof(d), r, y, dr, dh, pw, pb, gate, qw, dx, dy, dgate, dpw, dpb, dqw, dqb, ws, n, None)
    for change in (dict(gate=64), dict(dgate=64), dict(dy=64), dict(post=1), dict(dpw=64), dict(pre=0), dict(pre=0, dh=None), dict(dh=None), dict(r=None),
                   dict(lddh=15), dict(rows=-1)):
        assert call(**change) == 1, change
    assert call(dh=66) == 3 and call(cols=16385) == 2
    assert call(rows=0) == 0


def test_workspace_size(L):
    size = lambda gate=False, **k: nq.nq_block_norm_backward_workspace_bytes(desc(**k), gate)
    assert size(cols=0) == -1 and size(cols=16385) == -1
    assert size() > 0 and size() % 4 == 0
    assert size(rows=4096, gate=True) > size(rows=4096)              # a gate's sums are joined from several thread blocks
