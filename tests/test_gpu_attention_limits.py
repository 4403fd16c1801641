"""The attention operators at the ends of what they accept, against the definition in 64 bits."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from attention_reference import check
from test_gpu_prompt_attention import definition as prompt_definition, inputs, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads", [(2, 1), (3, 1)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 150, 2 ** 30])
def test_windows_that_hide_nothing_with_too_few_keys(window, heads, causal):
    """The distance of a row's last key from a window's first is below -2^31 here."""
    q, k, v = inputs(300 + 20, 100 + 20, *heads, 64)
    args = q, k, v, starts_of([300, 20]), starts_of([100, 20])
    got = nq.nq_prompt_attention(*args, causal=causal, window=window)
    assert torch.equal(got, nq.nq_prompt_attention(*args, causal=causal))
    want, bound = prompt_definition(q, k, v, [300, 20], [100, 20], causal, 0, 0.125)
    check(got, want, bound)
