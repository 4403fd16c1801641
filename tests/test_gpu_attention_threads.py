"""The attention calls from several threads at once, each on a stream of its own: the first calls of a process too."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = '''
import threading, torch
import paper_2506_17870_b200 as nq
from paper_2506_17870_b200.attention import rotary_angles
nq.lib()
n, faults = 300, []
starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
at = torch.arange(n, dtype=torch.int32, device="cuda")
angles = rotary_angles(n, 64)
table = torch.arange(19, dtype=torch.int32, device="cuda")[None]
xs = [torch.randn(n, 8 * 64, device="cuda").bfloat16() for _ in range(8)]
torch.cuda.synchronize()
start = threading.Barrier(8)

def once(x):
    c = nq.nq_kv_pages(*(torch.zeros(19, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    q, k = nq.nq_qk_norm_rotate(x, angles, at, q_heads=4, kv_heads=2, cache=c, slots=at, want_k=True)
    y = nq.nq_prompt_attention(q, k, x.view(n, 8, 64)[:, 6:], starts)
    kr, vr = nq.nq_kv_cache_read(c, table, starts, n)
    return y, nq.nq_prompt_attention(q, kr, vr, starts), nq.nq_paged_attention(q[-1:], c, table, starts[1:])

got = [None] * 8
def work(i):
    try:
        torch.cuda.set_device(0)
        with torch.cuda.stream(torch.cuda.Stream()):
            start.wait()
            got[i] = [once(xs[i]) for _ in range(20)]
            torch.cuda.current_stream().synchronize()
    except Exception as e:
        faults.append(e)

threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
assert not faults, faults
for i in range(8):
    want = once(xs[i])
    torch.cuda.synchronize()
    for out in got[i]:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
nq.nq_device_status()
print("threads agree")
'''


def test_first_calls_from_eight_threads():
    done = subprocess.run([sys.executable, "-c", PROGRAM], cwd=Path(__file__).resolve().parents[1], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "threads agree" in done.stdout, done.stderr[-2000:]
