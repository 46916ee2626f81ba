"""Weights of the cached keys where the tables of several sequences name the same pages: such a slot gets what all of them give.

Tolerance: each sequence's part as in tests/cache_weigh_util.py; they are added one after the other (a sequence's own in one addition for every 512
rows), each time with a rounding of at most 2^-24 of the new weight, since all summands are positive."""
import math

import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache
from tests.cache_util import routed
from tests.cache_weigh_util import weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("page,heads,B,common,length,new", [
    (16, (8, 2, 64), 24, 3, 100, 1),               # few rows
    (64, (28, 4, 128), 16, 4, 300, 2),
    (32, (16, 2, 128), 5, 10, 400, 70),            # blocks of rows
    (128, (8, 4, 64), 9, 2, 300, 40),
])
def test_common_pages_get_the_weights_of_all(kind, page, heads, B, common, length, new):
    Hq, Hkv, D = heads
    lengths = [length + 5 * b for b in range(B)]
    c = make_cache(kind, page, Hkv, D, lengths, 31)
    c.table[:, :common] = c.table[0, :common]
    for b in range(1, B):
        c.K[b][:common * page] = c.K[0][:common * page]
    N = B * new
    Q = torch.randn((N, Hq, D), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    d = routed(N, 0.7, 2)
    pool = (torch.rand((c.poolK.shape[0], Hkv, page), generator=torch.Generator().manual_seed(6)) * 1e-3).cuda()
    want, bound = pool.double(), torch.zeros_like(pool, dtype=torch.float64)
    most = max(lengths)
    p = l2a.params(B, new + 1, most, Hq, Hkv, D, 0)
    ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, N), dtype=torch.uint8, device="cuda")
    cu = torch.arange(0, N + 1, new, dtype=torch.int32, device="cuda")
    l2a.l2a_cache_weigh(p, c.handle, Q, cu, N, d, pool, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    additions = 0
    for b, (inc, off) in enumerate(weights(c, Q, [new] * B, d)):
        j = torch.arange(lengths[b], device="cuda")
        at, slot = c.table[b, j // page].long(), j % page
        fresh = j >= lengths[b] - new
        want[at[fresh], :, slot[fresh]] = 0
        want[at, :, slot] += inc
        bound[at, :, slot] += off
        additions += max(1, math.ceil(int(d[b * new:(b + 1) * new].sum()) * (Hq // Hkv) / 512))
    bound += additions * 2.0 ** -24 * want + 1e-36
    err = (pool.double() - want).abs()
    assert torch.isfinite(pool).all()
    assert bool((err <= bound).all()), f"{float((err / bound).max()):.3f} times the bound"
