"""Paged cache: NaN in a query row makes that row's result NaN, on every path, and no other row's."""
import pytest
import torch

from tests.cache_util import Cache, forward, routed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,lengths,new,W", [
    ((28, 4, 128), [60, 40], [1, 1], 100),               # one piece a sequence
    ((28, 4, 128), [9000, 700], [1, 1], 100),            # parts that are combined
    ((8, 1, 64), [9000, 700], [3, 2], 100),
    ((28, 4, 128), [700, 300], [40, 40], 100),           # chunks
    ((8, 1, 64), [9000, 300], [70, 40], 1000),
    ((32, 8, 128), [3000], [600], 100),
])
def test_nan_in_a_query_row(kind, heads, lengths, new, W):
    Hq, Hkv, D = heads
    c = Cache(kind, 64, Hkv, D, lengths, 28)
    N = sum(new)
    d = routed(N, 0.5, 3)
    d[0], d[N - 1] = 1, 0
    Q = torch.randn((N, Hq, D), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    want = forward(c, Hq, new, W, d=d, Q=Q)[0].clone()
    bad = torch.zeros((N, Hq), dtype=torch.bool, device="cuda")
    for t, h, e in ((0, 1, 3), (N - 1, Hq - 1, D - 1), (N // 2, 0, 0)):
        Q[t, h, e] = float("nan")
        bad[t, h] = True
    O = forward(c, Hq, new, W, d=d, Q=Q)[0]
    assert bool(O[bad].isnan().all())
    assert torch.equal(O[~bad], want[~bad])
