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
int group_in(int n, int length) {{ return nq::group_in(n, length); }}
long long wait_limit(long long one, int steps) {{ return nq::wait_limit(one, steps); }}
}}
''')
    subprocess.run(["g++", "-O2", "-ftrapv", "-shared", "-fPIC", "-o", str(library), str(source)], check=True)
    loaded = ctypes.CDLL(str(library))
    loaded.wait_limit.restype, loaded.wait_limit.argtypes = ctypes.c_longlong, (ctypes.c_longlong, ctypes.c_int)
    return loaded


@pytest.mark.parametrize("window", [0, 1, 100, MOST - 200, MOST - 1, MOST])
def test_window_start(ranges, window):
    for reach in (-MOST + 4096, -200, -1, 0, 1, 99, 100, 101, MOST - 4096, MOST):
        assert ranges.window_start(window, reach) == (max(0, reach - window) if window else 0)


@pytest.mark.parametrize("page", [16, 32, 48, 64, 128, 256, 512])
@pytest.mark.parametrize("tokens", [16, 32])
def test_no_page_is_asked_for_behind_the_table(ranges, page, tokens):
    """A warp of the single-token kernel asks for the pages of 32 groups of 16 tokens, from the one that its step starts at.  In the largest table
    that is accepted, the last sequence's last steps ask for none behind its columns, and for all that there are."""
    columns = MOST // page
    for length in (columns * page, columns * page - 1, columns * page - 17, 33):
        last = (length - 1) // 16
        for first in range(max(0, last - 40) // (tokens // 16) * (tokens // 16), last + 1, tokens // 16):
            for n in range(first, first + 32):
                asked = bool(ranges.group_in(n, length))
                assert asked == (16 * n < length)
                assert not asked or n // (page // 16) < columns
    assert not ranges.group_in(0, 0) and not ranges.group_in(0, -5) and ranges.group_in(0, 1)


def test_a_wait_for_many_steps_outlasts_them(ranges):
    """The tile without rows of a unit waits for the other's steps: 64 keys each, some 1650 cycles."""
    one = 2 ** 31
    for keys in (0, 64, 10 ** 6, 10 ** 8, MOST - 4096):
        steps = -(-keys // 64)
        assert ranges.wait_limit(one, steps) >= one // 2 + 5 * 1650 * steps
    assert ranges.wait_limit(one, 0) == ranges.wait_limit(one, -3) == one
    assert ranges.wait_limit(one, 8) < one + one // 1000                 # what is stuck is still given up after about a second
