"""The index-checking build (-DL2A_DEBUG) on 4-bit caches, the weights of cached keys and evictions, at small and odd sizes: no check fires, and the results are
within the tolerances of the normal build.  In a child process, so that this session keeps the normal library loaded."""
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
from tests.cache_e2m1_util import make_cache
from tests.cache_util import attention, check, forward, routed
from tests.cache_weigh_util import weigh
from tests.test_gpu_cache_evict import Target, run

HEADS = [(28, 4, 128), (12, 2, 64), (32, 8, 128)]
SIZES = [([300, 1, 900], [1, 1, 1]), ([300, 40], [9, 3]), ([1200, 400, 64], [300, 64, 1]), ([65, 64, 63, 129], [2, 0, 1, 5])]
for Hq, Hkv, D in HEADS:
    for lengths, new in SIZES:
        for page in (16, 128):
            c = make_cache("e2m1", page, Hkv, D, lengths, 5)
            d = routed(sum(new), 0.4, 5)
            O, Q = forward(c, Hq, new, 100, d=d)        # (reads the status word: a failed check fails it)
            check(O, *attention(c, Q, new, d, 100), f"{new}")
            x = torch.randn((sum(new), Hkv, D), device="cuda", dtype=torch.bfloat16)
            p = l2a.params(len(new), max(new), max(lengths), Hq, Hkv, D, 100)
            cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()
            l2a.l2a_cache_append(p, c.handle, x, x, cu, sum(new))
            out = torch.empty((2, len(new), max(lengths), Hkv, D), dtype=torch.bfloat16, device="cuda")
            l2a.l2a_cache_read(p, c.handle, None, out[0], out[1])
        for kind in ("bf16", "e4m3", "e2m1"):
            weigh(make_cache(kind, 32, Hkv, D, lengths, 6), Hq, new, routed(sum(new), 0.5, 1))      # (the same)
for kind in ("bf16", "e4m3", "e2m1"):
    for D in (64, 128):
        run(kind, 32, 16, 2, D, [9000, 1, 0, 130], [700, 1, 3, 129], 3, 40)
        lengths, keep = [20000, 7], [3000, 7]
        c = make_cache(kind, 64, 2, D, lengths, 3)
        t = Target(c, 3000, 64)
        p = l2a.params(2, 3000, 20000, 2, 2, D, 0)
        ws = torch.empty(l2a.l2a_cache_evict_workspace_bytes(p, c.handle), dtype=torch.uint8, device="cuda")
        w = torch.rand((c.poolK.shape[0], 2, 64), device="cuda")
        l2a.l2a_cache_evict(p, c.handle, w, torch.tensor(keep, dtype=torch.int32).cuda(), 4, 100, t.handle, t.w, t.lengths, None, ws)
        assert l2a.l2a_workspace_status(ws) == 0
torch.cuda.synchronize()
print("CACHE_DEBUG_OK")
"""


def test_debug_build_runs_long_lived_caches():
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], cwd=ROOT, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "CACHE_DEBUG_OK" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
