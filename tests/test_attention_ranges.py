"""The attention kernels' integer arithmetic at the ends of what they accept, on the CPU: their own header, compiled by itself."""
import ctypes
import subprocess
from pathlib import Path

import pytest

HEADER = Path(__file__).resolve().parents[1] / "paper_2506_17870_b200" / "csrc" / "nq_ranges.cuh"
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    folder = tmp_path_factory.mktemp("ranges")
    source, library = folder / "ranges.cpp", folder / "ranges.so"
    source.write_text(f'''#include "{HEADER}"
extern "C" {{
int window_start(int window, int reach) {{ return nq::window_start(window, reach); }}
}}
''')
    subprocess.run(["g++", "-O2", "-ftrapv", "-shared", "-fPIC", "-o", str(library), str(source)], check=True)
    return ctypes.CDLL(str(library))


@pytest.mark.parametrize("window", [0, 1, 100, MOST - 200, MOST - 1, MOST])
def test_window_start(ranges, window):
    for reach in (-MOST + 4096, -200, -1, 0, 1, 99, 100, 101, MOST - 4096, MOST):
        assert ranges.window_start(window, reach) == (max(0, reach - window) if window else 0)
