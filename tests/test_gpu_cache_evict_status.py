"""Eviction from a paged cache: the call leaves its status in the workspace, as all others do, whatever was there."""
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache
from tests.test_gpu_cache_evict import Target

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,keep", [([40, 17], [20, 3]), ([0, 5], [4, 0]), ([20000, 3], [700, 3])])
def test_status_of_a_call(lengths, keep):
    c = make_cache("e2m1", 64, 2, 64, lengths, 2)
    t = Target(c, max(keep), 32)
    p = l2a.params(2, max(keep), max(lengths), 2, 2, 64, 0)
    ws = torch.full((l2a.l2a_cache_evict_workspace_bytes(p, c.handle),), 0xA5, dtype=torch.uint8, device="cuda")
    w = torch.rand((c.poolK.shape[0], 2, 64), device="cuda")
    l2a.l2a_cache_evict(p, c.handle, w, torch.tensor(keep, dtype=torch.int32).cuda(), 1, 2, t.handle, t.w, t.lengths, None, ws)
    assert l2a.l2a_workspace_status(ws) == 0
    assert t.lengths.tolist() == [min(n, k) for n, k in zip(lengths, keep)]
