"""Weights of the cached keys: what a query row with NaN or infinities gives stays with the keys that it sees.  A row gives nothing to a key
behind its position, whatever its scores are, so that all other weights have the bits that they have with any other row in its place."""
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 128


def weigh(c, Q, new):
    w = torch.full((c.poolK.shape[0], HKV, c.page), 0.5, device="cuda")
    p = l2a.params(len(new), max(new), max(c.lengths), HQ, HKV, D, 0)
    ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, sum(new)), dtype=torch.uint8, device="cuda")
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()
    l2a.l2a_cache_weigh(p, c.handle, Q, cu, sum(new), None, w, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    return w


def check(kind, page, lengths, new, value):
    c = make_cache(kind, page, HKV, D, lengths, 21)
    Q = torch.randn((sum(new), HQ, D), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    want = weigh(c, Q, new)
    assert torch.isfinite(want).all()
    head, g = 5, 5 // (HQ // HKV)
    for token in sorted({0, new[0] // 2, new[0] - 1}):           # of the first sequence
        bad = Q.clone()
        bad[token, head] = value
        got = weigh(c, bad, new)
        j = torch.arange(lengths[0] - new[0] + token + 1, device="cuda")
        at, slot = c.table[0, j // page].long(), j % page
        if value != value:
            assert bool(got[at, g, slot].isnan().all()), f"token {token}: a weight of a key that the row sees is a number"
        seen = torch.zeros_like(want, dtype=torch.bool)
        seen[at, g, slot] = True
        assert torch.equal(got[~seen].view(torch.int32), want[~seen].view(torch.int32)), f"token {token}: a key that the row does not see"


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind,page,lengths,new", [("bf16", 16, [300, 100], [2, 1]), ("e4m3", 64, [300, 40], [7, 2]), ("e2m1", 32, [300, 40], [2, 2]),
                                                   ("e2m1", 64, [700, 40], [12, 2]), ("bf16", 64, [12, 40], [12, 2])])
def test_few_rows(kind, page, lengths, new, value):
    check(kind, page, lengths, new, value)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind,page,lengths,new", [("bf16", 16, [500, 100], [90, 30]), ("e4m3", 64, [1000, 40], [200, 2]),
                                                   ("e2m1", 128, [400, 300], [400, 20])])
def test_blocks_of_rows(kind, page, lengths, new, value):
    check(kind, page, lengths, new, value)
