"""The attention calls have no gradients: a backward pass through them ends with an error that says so, not with constants.  Tensors of the host
stand in for those of a GPU; the library does nothing."""
import pytest
import torch

from paper_2506_17870_b200 import binding
from test_attention_operand_devices import calls
from test_fp8_operand_devices import no_library  # noqa: F401

WHAT = [(0, "x"), (0, "q_weight"), (0, "k_weight"), (3, "q"), (4, "q"), (4, "k"), (4, "v")]


@pytest.fixture(autouse=True)
def library_that_does_nothing(no_library, monkeypatch):  # noqa: F811
    class Library:
        def __getattr__(self, name):
            return lambda *_: 4096 if name.endswith("workspace_bytes") else 0
    monkeypatch.setattr(binding, "lib", lambda: Library())


def outputs(y):
    return [t for t in (y if isinstance(y, tuple) else (y,)) if t is not None]


@pytest.mark.parametrize("which,name", WHAT)
def test_backward_passes_are_refused(which, name):
    call, good = list(calls())[which]
    good[name].requires_grad_()
    if which == 0:
        good["want_k"] = True
    tied = [t for t in outputs(call(**good)) if t.requires_grad]
    assert len(tied) == (2 if name == "x" else 1)
    for y in tied:
        with pytest.raises(RuntimeError, match="has no gradient"):
            y.float().sum().backward()


@pytest.mark.parametrize("which,name", WHAT)
def test_calls_without_gradients_stay_as_they_are(which, name):
    call, good = list(calls())[which]
    assert not any(t.requires_grad for t in outputs(call(**good)))
    call, good = list(calls())[which]
    good[name].requires_grad_()
    with torch.no_grad():
        assert not any(t.requires_grad for t in outputs(call(**good)))


@pytest.mark.parametrize("which", [3, 4])
def test_an_output_of_ones_own_is_what_comes_back(which):
    call, good = list(calls())[which]
    assert call(**good) is good["y_out"]
    good["q"].requires_grad_()
    assert call(**good) is good["y_out"] and good["y_out"].requires_grad
