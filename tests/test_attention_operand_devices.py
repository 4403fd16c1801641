"""Every operand of the attention calls has to lie on the first one's GPU, the cache and a workspace too: refused on the host, before
anything is handed to the library.  Tensors of the host stand in for those of two GPUs; the library is not there."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from test_fp8_operand_devices import OnGpu, OnOther, Reached, elsewhere, no_library, refused  # noqa: F401

BF16, I32 = torch.bfloat16, torch.int32


def zeros(*shape, dtype=BF16):
    return torch.zeros(*shape).to(dtype).as_subclass(OnGpu)


def pages(kind=OnGpu):
    t = lambda *s, dtype: torch.zeros(*s).to(dtype).as_subclass(kind)
    return nq.nq_kv_pages(t(3, 2, 16, 64, dtype=torch.int8), t(3, 2, 16, 64, dtype=torch.int8), t(3, 2, 16, dtype=torch.float32), t(3, 2, 16, dtype=torch.float32))


@pytest.mark.parametrize("name", ["k", "v", "ks", "vs"])
def test_a_cache_is_in_one_place(name):
    good = dict(k=zeros(3, 2, 16, 64, dtype=torch.int8), v=zeros(3, 2, 16, 64, dtype=torch.int8), ks=zeros(3, 2, 16, dtype=torch.float32),
                vs=zeros(3, 2, 16, dtype=torch.float32))
    nq.nq_kv_pages(**good)
    for t in elsewhere(good[name]):
        with pytest.raises(ValueError):
            nq.nq_kv_pages(**{**good, name: t})


def calls():
    table, lengths, slots = zeros(2, 3, dtype=I32), zeros(2, dtype=I32), zeros(5, dtype=I32)
    yield lambda **k: nq.nq_qk_norm_rotate(k.pop("x"), k.pop("angles"), k.pop("positions"), q_heads=4, kv_heads=2, **k), dict(
        x=zeros(5, 512), angles=zeros(9, 64, dtype=torch.float32), positions=zeros(5, dtype=I32), q_weight=zeros(64, dtype=torch.float32),
        k_weight=zeros(64, dtype=torch.float32), slots=slots, cache=pages())
    yield lambda **k: nq.nq_kv_cache_write(**k), dict(cache=pages(), k=zeros(5, 2, 64), v=zeros(5, 2, 64), slots=slots)
    yield lambda **k: nq.nq_kv_cache_read(**k, rows=7), dict(cache=pages(), table=table, starts=zeros(3, dtype=I32), k_out=zeros(7, 2, 64), v_out=zeros(7, 2, 64))
    yield lambda **k: nq.nq_paged_attention(**k), dict(q=zeros(2, 4, 64), cache=pages(), table=table, lengths=lengths, y_out=zeros(2, 4, 64),
                                                       workspace=zeros(4096, dtype=torch.uint8))
    yield lambda **k: nq.nq_prompt_attention(**k), dict(q=zeros(5, 4, 64), k=zeros(7, 2, 64), v=zeros(7, 2, 64), starts_q=zeros(3, dtype=I32),
                                                        starts_k=zeros(3, dtype=I32), y_out=zeros(5, 4, 64))


@pytest.mark.parametrize("which", range(5))
def test_operands(which):
    call, good = list(calls())[which]
    for name in good:
        if name == "cache":
            with pytest.raises(ValueError, match="cuda:1"):
                call(**{**good, "cache": pages(OnOther)})
        else:
            refused(call, good, name)


@pytest.mark.parametrize("which,name,bad", [
    (0, "positions", zeros(4, dtype=I32)), (0, "positions", zeros(5, dtype=torch.int64)), (0, "slots", zeros(6, dtype=I32)), (0, "angles", zeros(64, dtype=torch.float32)),
    (0, "x", zeros(5, 511)), (0, "x", zeros(5, 384)), (0, "q_weight", zeros(32, dtype=torch.float32)), (0, "slots", None), (0, "angles", None),
    (1, "k", zeros(5, 3, 64)), (1, "v", zeros(4, 2, 64)), (1, "v", zeros(5, 2, 64, dtype=torch.float32)), (1, "slots", zeros(4, dtype=I32)), (1, "k", zeros(5, 128)),
    (2, "table", zeros(3, dtype=I32)), (2, "table", zeros(2, 3, dtype=torch.int64)), (2, "starts", zeros(2, dtype=I32)), (2, "k_out", zeros(6, 2, 64)), (2, "v_out", None),
    (3, "q", zeros(2, 4, 64, dtype=torch.float32)), (3, "q", zeros(2, 4, 128)), (3, "table", zeros(3, 3, dtype=I32)), (3, "lengths", zeros(3, dtype=I32)),
    (3, "lengths", zeros(2, dtype=torch.int64)), (3, "y_out", zeros(2, 4, 64, dtype=torch.float32)),
    (4, "k", zeros(7, 2, 128)), (4, "v", zeros(6, 2, 64)), (4, "q", zeros(5, 4, 64, dtype=torch.float16)), (4, "starts_k", zeros(4, dtype=I32)),
    (4, "starts_q", zeros(3, dtype=torch.int64)), (4, "y_out", zeros(5, 2, 64)), (4, "starts_q", zeros(3, 1, dtype=I32))])
def test_shapes_and_types(which, name, bad):
    call, good = list(calls())[which]
    with pytest.raises(ValueError):
        call(**{**good, name: bad})


def test_strides():
    call, good = list(calls())[4]
    with pytest.raises(Reached):
        call(**{**good, "q": zeros(5, 9, 64)[:, 2:6]})
    for q in (zeros(5, 64, 4).transpose(1, 2), zeros(4, 5, 64).transpose(0, 1), zeros(1, 4, 64).expand(5, 4, 64)):
        with pytest.raises(ValueError):
            call(**{**good, "q": q})
