"""Refusals of the attention entry points that need no GPU: they come before any CUDA call."""
import ctypes

import pytest
import torch

import paper_2506_17870_b200 as nq
from paper_2506_17870_b200 import build as nq_build


@pytest.fixture(scope="module")
def L():
    nq_build.build()
    return nq.lib()


class Pages(ctypes.Structure):
    _fields_ = nq.nq_kv_pages._fields_


def pages(**k):
    base = dict(k=64, v=64, ks=None, vs=None, pages=4, page_size=16, kv_heads=2, head_dim=64, dtype=1)
    return Pages(**{**base, **k})


BAD_PAGES = [(dict(pages=-1), 1), (dict(page_size=0), 1), (dict(kv_heads=0), 1), (dict(dtype=0), 1), (dict(dtype=4), 1), (dict(k=None), 1), (dict(v=None), 1),
             (dict(ks=64), 1), (dict(vs=64), 1), (dict(dtype=2), 1), (dict(dtype=3, ks=64), 1), (dict(head_dim=96), 2), (dict(head_dim=256), 2), (dict(page_size=24), 2),
             (dict(page_size=32784), 2), (dict(pages=1 << 28), 2), (dict(kv_heads=65537), 2), (dict(k=72), 3), (dict(v=8), 3), (dict(dtype=2, ks=66, vs=64), 3)]


@pytest.mark.parametrize("change,status", BAD_PAGES)
def test_caches(L, change, status):
    p = pages(**change)
    at = ctypes.addressof(p)
    assert L.nq_kv_cache_write(at, 64, 128, 64, 128, 1, 64, 3, None) == status
    assert L.nq_kv_cache_read(at, 64, 4, 4, 64, 2, 64, 128, 64, 128, 1, 3, None) == status
    assert L.nq_paged_attention(at, 64, 256, 4, 64, 4, 4, 64, 2, 0, 0.125, 64, 256, 64, 1 << 30, None) == status
    assert L.nq_paged_attention_workspace_bytes(at, 4, 2, 4) == -1
    d = nq.nq_qk_desc(3, 512, 256, 128, 0, 1, 1, 4, p.kv_heads, p.head_dim, 0, 0, 0, 1e-6)
    if p.kv_heads > 0 and p.kv_heads < 9 and p.head_dim in (64, 128):
        assert L.nq_qk_norm_rotate(ctypes.addressof(d), 64, None, None, None, None, 64, None, at, 64, None) == status


def test_no_cache(L):
    assert L.nq_kv_cache_write(None, 64, 128, 64, 128, 1, 64, 3, None) == 1
    assert L.nq_kv_cache_read(None, 64, 4, 4, 64, 2, 64, 128, 64, 128, 1, 3, None) == 1
    assert L.nq_paged_attention(None, 64, 256, 4, 64, 4, 4, 64, 2, 0, 0.125, 64, 256, 64, 1 << 30, None) == 1
    assert L.nq_paged_attention_workspace_bytes(None, 4, 2, 4) == -1


def test_qk_norm_rotate(L):
    def call(x=64, qw=None, kw=None, angles=64, positions=64, q=64, k=64, cache=None, slots=None, **change):
        base = dict(tokens=3, ldx=512, ldq=256, ldk=128, angle_rows=9, x_dtype=1, y_dtype=1, q_heads=4, kv_heads=2, head_dim=64, rotary_dim=64, norm=1, neighbours=0,
                    eps=1e-6)
        d = nq.nq_qk_desc(**{**base, **change})
        return L.nq_qk_norm_rotate(ctypes.addressof(d), x, qw, kw, angles, positions, q, k, cache, slots, None)
    for change in (dict(tokens=-1), dict(q_heads=-1), dict(kv_heads=-1), dict(angle_rows=-1), dict(rotary_dim=-16), dict(eps=-1.0), dict(eps=float("nan")), dict(x_dtype=2),
                   dict(y_dtype=3), dict(norm=2), dict(norm=0, qw=64), dict(norm=0, kw=64), dict(slots=64), dict(x=None), dict(q=None), dict(k=None), dict(ldx=383),
                   dict(ldq=255), dict(ldk=127), dict(positions=None), dict(angles=None), dict(angle_rows=0)):
        assert call(**change) == 1, change
    for change in (dict(head_dim=32), dict(head_dim=256), dict(rotary_dim=24), dict(rotary_dim=80), dict(q_heads=65537), dict(angle_rows=1 << 31)):
        assert call(**change) == 2, change
    for change in (dict(x=72), dict(q=72), dict(k=72), dict(qw=68), dict(kw=72), dict(angles=72), dict(positions=66), dict(ldx=516), dict(ldq=260), dict(ldk=132),
                   dict(x_dtype=0, ldx=513)):
        assert call(**change) == 3, change
    p = pages()
    at = ctypes.addressof(p)
    assert call(cache=at) == 1 and call(cache=at, slots=64, kv_heads=1) == 1 and call(cache=at, slots=64, ldx=448) == 1 and call(cache=at, slots=66) == 3
    assert call(tokens=0) == 0 and call(tokens=0, x=None, q=None, k=None) == 0 and call(q_heads=0, kv_heads=0) == 0
    assert L.nq_qk_norm_rotate(None, 64, None, None, None, None, 64, 64, None, None, None) == 1


def test_write_and_read(L):
    p = pages()
    at = ctypes.addressof(p)
    write = lambda k=64, ldk=128, v=64, ldv=128, t=1, slots=64, n=3: L.nq_kv_cache_write(at, k, ldk, v, ldv, t, slots, n, None)
    for change in (dict(k=None), dict(v=None), dict(slots=None), dict(ldk=127), dict(ldv=127), dict(t=2), dict(n=-1)):
        assert write(**change) == 1, change
    for change in (dict(k=72), dict(v=72), dict(slots=66), dict(ldk=132), dict(ldv=130), dict(t=0, ldv=129)):
        assert write(**change) == 3, change
    assert write(n=0, k=None) == 0 and write(n=1 << 40) == 2
    read = lambda table=64, ld=4, cols=4, starts=64, seqs=2, k=64, ldk=128, v=64, ldv=128, t=1, rows=3: L.nq_kv_cache_read(
        at, table, ld, cols, starts, seqs, k, ldk, v, ldv, t, rows, None)
    for change in (dict(table=None), dict(ld=3), dict(cols=-1), dict(starts=None), dict(seqs=-1), dict(k=None), dict(v=None), dict(ldk=127), dict(ldv=127), dict(t=3), dict(rows=-1)):
        assert read(**change) == 1, change
    for change in (dict(table=66), dict(starts=66), dict(k=72), dict(v=72), dict(ldk=132), dict(ldv=132)):
        assert read(**change) == 3, change
    assert read(rows=0, k=None) == 0 and read(seqs=0, starts=None) == 0 and read(rows=1 << 31) == 2


def test_paged_attention(L):
    p = pages()
    at = ctypes.addressof(p)
    call = lambda q=64, ldq=256, heads=4, table=64, ld=4, cols=4, lengths=64, seqs=2, window=0, scale=0.125, y=64, ldy=256, ws=64, n=1 << 30: L.nq_paged_attention(
        at, q, ldq, heads, table, ld, cols, lengths, seqs, window, scale, y, ldy, ws, n, None)
    for change in (dict(q=None), dict(ldq=255), dict(heads=3), dict(heads=0), dict(heads=-2), dict(table=None), dict(ld=3), dict(cols=-1), dict(lengths=None), dict(seqs=-1),
                   dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(y=None), dict(ldy=255)):
        assert call(**change) == 1, change
    for change in (dict(q=72), dict(ldq=260), dict(table=66), dict(lengths=66), dict(y=72), dict(ldy=260), dict(ws=72)):
        assert call(**change) == 3, change
    assert call(ws=None) == 4 and call(n=16) == 4
    assert call(heads=65538) == 2 and call(cols=1 << 28, ld=1 << 28) == 2 and call(seqs=1 << 30) == 2
    assert call(seqs=0, q=None) == 0
    size = lambda heads, seqs, cols: L.nq_paged_attention_workspace_bytes(at, heads, seqs, cols)
    assert size(3, 2, 4) == -1 and size(4, -1, 4) == -1
    assert 0 < size(4, 1, 1) <= size(4, 2, 4) <= size(4, 64, 4096) < 32 << 20 and size(4, 0, 0) > 0


def test_python_refusals():
    """Shapes, types and places that the Python calls check themselves; on host tensors, so that nothing can run."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="bfloat16, float8_e4m3fn or int8"):
        nq.nq_kv_pages(torch.zeros(1, 1, 16, 64), torch.zeros(1, 1, 16, 64))
    with pytest.raises(ValueError, match="pages, kv_heads"):
        nq.nq_kv_pages(bf(1, 1, 16, 64), bf(1, 1, 16, 128))
    with pytest.raises(ValueError, match="ks and vs go with"):
        nq.nq_kv_pages(bf(1, 1, 16, 64), bf(1, 1, 16, 64), torch.zeros(1, 1, 16), torch.zeros(1, 1, 16))
    with pytest.raises(ValueError, match="ks and vs go with"):
        nq.nq_kv_pages(torch.zeros(1, 1, 16, 64, dtype=torch.int8), torch.zeros(1, 1, 16, 64, dtype=torch.int8))
    with pytest.raises(ValueError, match="CUDA"):
        nq.nq_kv_pages(bf(1, 1, 16, 64), bf(1, 1, 16, 64))
    with pytest.raises(ValueError, match="CUDA"):
        nq.nq_qk_norm_rotate(bf(3, 256), None, None, q_heads=2, kv_heads=1)
    with pytest.raises(ValueError, match="\\[rows, cols\\]"):
        nq.nq_qk_norm_rotate(bf(3, 2, 128), None, None, q_heads=2, kv_heads=1)


def test_prompt_attention(L):
    def call(q=64, k=64, v=64, sq=64, sk=64, y=64, **change):
        base = dict(seqs=2, rows_q=9, rows_k=11, ldq=256, ldk=128, ldv=128, ldy=256, q_heads=4, kv_heads=2, head_dim=64, causal=1, window=0, scale=0.125)
        d = nq.nq_prompt_desc(**{**base, **change})
        return L.nq_prompt_attention(ctypes.addressof(d), q, k, v, sq, sk, y, None)
    for change in (dict(seqs=-1), dict(rows_q=-1), dict(rows_k=-1), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=3), dict(window=-1), dict(scale=0.0), dict(scale=-1.0),
                   dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None), dict(k=None), dict(v=None), dict(sq=None), dict(sk=None), dict(y=None), dict(ldq=255),
                   dict(ldk=127), dict(ldv=127), dict(ldy=255)):
        assert call(**change) == 1, change
    for change in (dict(head_dim=96), dict(head_dim=256), dict(rows_q=1 << 31), dict(rows_k=1 << 31), dict(seqs=1 << 30), dict(q_heads=65538)):
        assert call(**change) == 2, change
    for change in (dict(q=72), dict(k=72), dict(v=72), dict(y=72), dict(sq=66), dict(sk=66), dict(ldq=260), dict(ldk=132), dict(ldv=132), dict(ldy=260)):
        assert call(**change) == 3, change
    assert call(seqs=0, q=None) == 0 and call(rows_q=0, q=None) == 0
    assert L.nq_prompt_attention(None, 64, 64, 64, 64, 64, 64, None) == 1
