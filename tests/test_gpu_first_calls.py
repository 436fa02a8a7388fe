"""GPU tests of first calls: a host thread whose first CUDA call is one of the library's."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = r"""
import sys, threading
sys.path.insert(0, %r)
import torch
from paper_2608_08097_b200 import binding as L
torch.cuda.init()
N = 16
dims = L.Dims(1, 4, 1, 4)
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
bf = dict(dtype=torch.bfloat16, device="cuda")
q, kv, pool = torch.ones((1, 3, 4, 128), **bf), torch.ones((1, 3, 1, 2, 128), **bf), torch.ones((4, 2, 16, 128), **bf)
parent, nodes, slot, blk, lens = i32([[-1, 0, 0]]), i32([3]), i32([[[0, 1, 2, 3]]]), i32([[[0, 1, -1, -1]]]), i32([20])
outs = [torch.zeros_like(q) for _ in range(N)]
streams = [torch.cuda.Stream() for _ in range(N)]
L._calls()
torch.cuda.synchronize()
gate, failed = threading.Barrier(N), []
def work(i):
    gate.wait()
    try:
        L.tree_attn(dims, q, kv, parent, nodes, pool, slot, blk, lens, 0.1, outs[i], stream=streams[i])
    except Exception as e:
        failed.append(repr(e))
threads = [threading.Thread(target=work, args=(i,)) for i in range(N)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert not failed, failed
assert all((o == 1).all() for o in outs)
print("ok")
"""


def test_threads_whose_first_call_is_the_librarys():
    """Sixteen threads that have no CUDA context yet call the attention at the same time, each on a stream of its own."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import build
    build.build()
    for _ in range(3):
        r = subprocess.run([sys.executable, "-c", CODE % ROOT], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-1000:] + r.stderr[-2000:]
