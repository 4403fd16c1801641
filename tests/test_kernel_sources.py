"""Rules of the kernels' sources that no run can show: a violation may work for years and then hang."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2506_17870_b200" / "csrc"


def unordered(text):
    """Lines of warp-wide tensor-memory instructions (tcgen05 loads and their wait, `.sync.aligned`) that follow a barrier wait,
    in which each lane spins by itself, without a vote or __syncwarp() that brings the lanes together in between."""
    apart, found = False, []
    for n, line in enumerate(text.splitlines(), 1):
        for word in re.findall(r"mbar_wait\w*\(|__all_sync\(|__syncwarp\(|__syncthreads\(|tmem_ld\w*\(", line.split("//")[0]):
            if word.startswith("mbar_wait"):
                apart = True
            elif word.startswith("tmem_ld"):
                if apart:
                    found.append(n)
            else:
                apart = False
    return found


def test_the_rule_itself():
    assert unordered("ok = mbar_wait(a);\ntmem_ld_wait();") == [2]
    assert unordered("ok = mbar_wait(a); ok = __all_sync(m, ok);\ntmem_ld_32x32(t, r);\ntmem_ld_wait();") == []


@pytest.mark.parametrize("path", sorted(p.name for p in CSRC.iterdir() if p.suffix in (".cu", ".cuh") and p.name != "nq_sm100.cuh"))
def test_lanes_come_together_before_tensor_memory(path):
    assert unordered((CSRC / path).read_text()) == []
