"""What no run of the attention calls shows: they keep nothing between calls that two threads could write at once (Python lets go of its lock
while the library runs)."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2506_17870_b200" / "csrc"


@pytest.mark.parametrize("name", ["nq_runtime.cu", "nq_kv_cache.cu", "nq_kv_cache.cuh", "nq_paged_attention.cu", "nq_prompt_attention.cu"])
def test_statics_are_atomic(name):
    text = re.sub(r"//[^\n]*", "", (CSRC / name).read_text())
    kept = [line.strip() for line in text.splitlines() if re.match(r"\s*static\s+(?!constexpr|const\b)[^(]*[;=]", line)]
    assert all(line.startswith("static std::atomic<") for line in kept), kept
