"""Every operand of the e4m3 and block-norm calls has to lie on the first one's GPU, and a workspace too: refused on the host,
before anything is handed to the library.  Tensors of the host stand in for those of two GPUs; the library is not there."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from paper_2506_17870_b200 import binding

F8 = torch.float8_e4m3fn


class OnGpu(torch.Tensor):
    index = 0
    is_cuda = True

    def get_device(self):
        return self.index


class OnOther(OnGpu):
    index = 1


class Reached(Exception):
    pass


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    class Library:
        def __getattr__(self, name):
            def call(*_):
                if name.endswith("workspace_bytes"):
                    return 4096
                raise Reached(name)
            return call
    monkeypatch.setattr(binding, "lib", lambda: Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape).to(dtype).as_subclass(OnGpu)


def elsewhere(t):
    """The same on the other GPU, and on the host."""
    plain = t.as_subclass(torch.Tensor)
    return [plain.clone().as_subclass(OnOther), plain.clone()]


def refused(call, good, name):
    with pytest.raises(Reached):                                   # the call itself is in order
        call(**good)
    for t in elsewhere(good[name]):
        with pytest.raises(ValueError):
            call(**{**good, name: t})


@pytest.mark.parametrize("name", ["a", "sa", "b", "sb", "bias", "y_out"])
@pytest.mark.parametrize("K", [256, 200])                          # dense, and with a pitch
def test_product(name, K):
    pitched = lambda rows: zeros(rows, 256, dtype=F8)[:, :K]
    good = dict(a=pitched(32), sa=zeros(2, 32), b=pitched(64), sb=zeros(2, 1), bias=zeros(64), y_out=zeros(32, 64))
    refused(nq.nq_fp8_gemm, good, name)


def test_quantiser():
    refused(nq.nq_fp8_quantize, dict(x=zeros(4, 64)), "x")


VECTORS = ("post_weight", "post_bias", "pre_weight", "pre_bias")


@pytest.mark.parametrize("name", ("x", "y", "gate", "r_out") + VECTORS)
def test_norm(name):
    good = dict(x=zeros(8, 64), y=zeros(8, 64), post=2, pre=2, gate=zeros(1, 64), r_out=zeros(8, 64), **{v: zeros(64) for v in VECTORS})
    refused(nq.nq_block_norm, good, name)


@pytest.mark.parametrize("name", ("r", "y", "dr", "dh", "gate", "workspace") + VECTORS)
def test_norm_backward(name):
    good = dict(r=zeros(8, 64), y=zeros(8, 64), dr=zeros(8, 64), dh=zeros(8, 64), post=2, pre=2, gate=zeros(1, 64),
                workspace=zeros(4096, dtype=torch.uint8), **{v: zeros(64) for v in VECTORS})
    refused(nq.nq_block_norm_backward, good, name)


def test_workspace_layout():
    good = dict(r=zeros(8, 64), dh=zeros(8, 64))
    with pytest.raises(ValueError):
        nq.nq_block_norm_backward(**good, workspace=zeros(8192, dtype=torch.uint8)[::2])
    with pytest.raises(Reached):
        nq.nq_block_norm_backward(**good, workspace=zeros(1024))
