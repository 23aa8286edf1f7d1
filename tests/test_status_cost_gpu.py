"""What gs_stream_status costs programs that do not call cross attention."""
import pathlib
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

COUNT = """
import sys, torch
sys.path.insert(0, {root!r})
from torch.profiler import profile, ProfilerActivity
from paper_2608_01528_gb300 import gramspace as gs
C = (torch.randint(0, 2, (40, 512)) * 2 - 1).float().cuda()

def copies():
    with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as p:
        gs.stream_status()
    return sum(e.count for e in p.key_averages() if e.key == "cudaMemcpyFromSymbol")

b = gs.build_basis(C)
gs.project_similarity(b, C)
copies()                      # (a profiler's first use records nothing)
before = copies()
Q, K = (torch.randn(2, n, 4, 64).bfloat16().cuda() for n in (40, 90))
o = gs.cross_attention(Q, K, K, want_lse=True)
forward = copies()
gs.cross_attention_backward(Q, K, K, o["O"], o["lse"], o["O"])
print("copies", before, forward, copies())
"""


def test_error_words_read(gs):
    """Six words, each by a blocking copy, as before cross attention had words of its own; those are read by a process
    that has launched its kernels."""
    root = str(pathlib.Path(__file__).resolve().parent.parent)
    r = subprocess.run([sys.executable, "-c", COUNT.format(root=root)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split()[-3:] == ["6", "7", "8"], r.stdout
