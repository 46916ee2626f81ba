"""Paged cache, bounds of the host above what the device's lists hold: a token axis longer than the list's last entry, Lq and Lk above
the actual ones, captured steps whose list changes.  Tolerance and definition: tests/cache_util.py."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import Cache, attention, check, routed

pytestmark = pytest.mark.gpu


def tokens(new):
    return torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()


def loose(cache, Hq, new, W, n_tokens, Lq, Lk, d, Q):
    """O of a call with these bounds, 3 in every element before it."""
    p = l2a.params(len(new), Lq, Lk, Hq, cache.Hkv, cache.D, W)
    ws = torch.full((l2a.l2a_cache_workspace_bytes(p, cache.handle, n_tokens),), 0xA5, dtype=torch.uint8, device="cuda")
    O = torch.full((n_tokens, Hq, cache.D), 3.0, dtype=torch.bfloat16, device="cuda")
    l2a.l2a_cache_forward(p, cache.handle, Q, tokens(new), n_tokens, d, O, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    return O


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,lengths,new,n_tokens,Lq,Lk", [
    ((28, 4, 128), [700, 300], [200, 1], 400, 200, 700),          # as many rows as there can be, the second sequence of few
    ((28, 4, 128), [700, 300], [1, 1], 400, 200, 4096),           # ... and both
    ((28, 4, 128), [700], [3], 600, 600, 700),                    # one sequence
    ((8, 1, 128), [500, 90, 20], [0, 30, 2], 300, 100, 500),
    ((4, 4, 64), [300, 40], [17, 16], 34, 17, 300),
    ((28, 4, 128), [700, 300, 50], [200, 1, 0], 260, 230, 5000),  # between
    ((28, 4, 128), [700, 300], [1, 1], 7, 5, 4096),               # bounds of drafted tokens
    ((32, 8, 128), [700, 300], [1, 0], 2, 1, 9000),               # a sequence that has left
    ((80, 1, 64), [300, 20], [2, 1], 14, 7, 300),                 # more heads of a group than the path of few rows takes
])
def test_bounds_above_the_actual_values(kind, heads, lengths, new, n_tokens, Lq, Lk):
    Hq, Hkv, D = heads
    c = Cache(kind, 16, Hkv, D, lengths, 31, per=-(-Lk // 16))
    N = sum(new)
    Q = torch.randn((n_tokens, Hq, D), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    d = routed(n_tokens, 0.6, 2)
    O = loose(c, Hq, new, 100, n_tokens, Lq, Lk, d, Q)
    assert bool((O[N:] == 3).all()), "rows of no sequence"
    check(O[:N], *attention(c, Q[:N], new, d[:N], 100), f"{kind} {heads} new {new} of {n_tokens}")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_captured_step_follows_its_list(kind):
    """One captured call over a token axis of fixed size, replayed as the list shrinks, empties and fills up."""
    Hq, Hkv, D, W, n_tokens = 28, 4, 128, 64, 400
    lengths = [700, 450]
    c = Cache(kind, 32, Hkv, D, lengths, 14)
    p = l2a.params(2, 200, 700, Hq, Hkv, D, W)
    ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, c.handle, n_tokens), dtype=torch.uint8, device="cuda")
    Q = torch.randn((n_tokens, Hq, D), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    d = routed(n_tokens, 0.5, 8)
    O = torch.empty_like(Q)
    cu = tokens([200, 200])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        l2a.l2a_cache_forward(p, c.handle, Q, cu, n_tokens, d, O, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l2a.l2a_cache_forward(p, c.handle, Q, cu, n_tokens, d, O, ws)
    for new in ([200, 200], [200, 1], [1, 1], [0, 3], [0, 0], [57, 199]):
        cu.copy_(tokens(new))
        O.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert l2a.l2a_workspace_status(ws) == 0
        N = sum(new)
        assert bool((O[N:] == 3).all())
        check(O[:N], *attention(c, Q[:N], new, d[:N], W), f"replay of {new}")
