"""The bounds-check build over the packed cache, in a process of its own because a process loads one build of the library."""
import json
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_source_pages_and_a_packed_engine_in_the_checked_build():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import build
    env = dict(os.environ, OASIS_LIB=build.build(checked=True))
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "packed_engine_checked_worker.py")], env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert json.loads(r.stdout.strip().splitlines()[-1])["ok"]
