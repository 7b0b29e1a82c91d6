"""Host threads that make a process's first calls of an operator at the same time, each with a size of its own and on its own stream: every
call goes through and gives what a single thread gets."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = """
import sys
sys.path[:0] = [%r, %r]
import threading
import torch
import paper_2109_09868_b200 as ap
from test_hosted_more_cpu import BLOCK_NORM

lib = ap.load()
g = torch.Generator().manual_seed(1)
shapes = [(T, N) for T in (2000, 3) for N in (520, 1000, 2048, 4096, 8192, 12000)]  # over the ring, and directly
calls = []
for T, N in shapes:
    r, y = (torch.randn((T, N), generator=g).cuda() for _ in range(2))
    w = torch.randn((4, N), generator=g).cuda()
    ro, x = torch.zeros_like(r), torch.zeros_like(r)
    args = BLOCK_NORM.pack(T, N, 1, 1, 2, 2, 0, 1.0, 1.0, 1e-6, 0, r.data_ptr(), N, y.data_ptr(), N, 0, 0, 0, *[w[i].data_ptr() for i in range(4)],
                           ro.data_ptr(), N, x.data_ptr(), N)
    calls.append((args, torch.cuda.Stream(), ro, x, (r, y, w)))
torch.cuda.synchronize()
codes, start = [None] * len(calls), threading.Barrier(len(calls))

def work(i):
    start.wait()
    codes[i] = [lib.approxifer_block_norm(calls[i][0], calls[i][1].cuda_stream) for _ in range(3)]

threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert all(c == [0, 0, 0] for c in codes), codes
for args, stream, ro, x, _ in calls:
    got = ro.clone(), x.clone()
    ro.zero_(), x.zero_()
    torch.cuda.synchronize()
    assert lib.approxifer_block_norm(args, stream.cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(ro, got[0]) and torch.equal(x, got[1])
print("all alike")
"""


def test_first_calls_of_different_widths_from_several_threads():
    done = subprocess.run([sys.executable, "-c", PROGRAM % (os.path.dirname(HERE), HERE)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "all alike" in done.stdout, done.stderr
