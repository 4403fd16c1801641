"""What the attention calls refuse on the host rather than answer for something else.  Tensors of the host stand in for those of a GPU; the
library is not there."""
import pytest
import torch

import paper_2506_17870_b200 as nq
from test_attention_operand_devices import calls
from test_fp8_operand_devices import Reached, no_library  # noqa: F401

ROTATE, WRITE, READ, TOKEN, PROMPT = range(5)


@pytest.mark.parametrize("which", [TOKEN, PROMPT])
def test_windows_past_32_bits(which):
    call, good = list(calls())[which]
    for window in (2 ** 31, 2 ** 32 + 5, 2 ** 64, -2 ** 32 + 5):
        with pytest.raises(ValueError, match="window"):
            call(**good, window=window)
    for window in (0, 5, 2 ** 31 - 1):
        with pytest.raises(Reached):
            call(**good, window=window)
