"""The index-checking build (-DL2A_DEBUG) on the calls of the paged cache: no check fires, and the results are those of the normal build's
tolerance.  In a child process, so that this session keeps the normal library loaded."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys
sys.path.insert(0, sys.argv[1])
import torch
from paper_2603_17484_b200 import build, l2a
l2a.LIB_PATH = build.build_lib(debug=True)
assert "debug" in l2a.version()
from tests.cache_util import Cache, attention, check, forward, routed
for kind in ("e4m3", "bf16"):
    for lengths, new in (([300, 1, 900], [1, 1, 1]), ([300, 40], [9, 3]), ([1200, 400, 64], [300, 64, 1])):
        c = Cache(kind, 32, 4, 128, lengths, 5)
        d = routed(sum(new), 0.4, 5)
        O, Q = forward(c, 28, new, 100, d=d)            # (reads the status word: a failed check fails it)
        check(O, *attention(c, Q, new, d, 100), f"{kind} {new}")
        x = torch.randn((sum(new), 4, 128), device="cuda", dtype=torch.bfloat16)
        p = l2a.params(len(new), max(new), max(lengths), 28, 4, 128, 100)
        cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()
        l2a.l2a_cache_append(p, c.handle, x, x, cu, sum(new))
torch.cuda.synchronize()
print("CACHE_DEBUG_OK")
"""


def test_debug_build_runs_the_cache():
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "CACHE_DEBUG_OK" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
