"""Paged cache: an 8-bit chunk with a workspace that has room for the decoded copy, and with one that has none: the same bits."""
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import Cache, attention, check, routed
from tests.test_gpu_cache_bounds import tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,lengths,new", [((28, 4, 128), [2000, 70], [300, 70]), ((8, 1, 64), [700], [200])])
def test_with_and_without_a_copy(heads, lengths, new):
    Hq, Hkv, D = heads
    c = Cache("e4m3", 32, Hkv, D, lengths, 29)
    plain = Cache("bf16", 32, Hkv, D, lengths, 29)
    N = sum(new)
    p = l2a.params(len(new), max(new), max(lengths), Hq, Hkv, D, 200)
    full, least = (l2a.l2a_cache_workspace_bytes(p, x.handle, N) for x in (c, plain))
    assert full > least
    Q = torch.randn((N, Hq, D), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    d = routed(N, 0.4, 1)
    out = []
    for size in (full, full - 1, least):
        ws = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        O = torch.full_like(Q, float("nan"))
        l2a.l2a_cache_forward(p, c.handle, Q, tokens(new), N, d, O, ws[:size])
        torch.cuda.synchronize()
        assert l2a.l2a_workspace_status(ws) == 0 and bool((ws[size:] == 0xA5).all())
        out.append(O)
    check(out[0], *attention(c, Q, new, d, 200), "with a copy")
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
    with pytest.raises(l2a.L2AError):
        l2a.l2a_cache_forward(p, c.handle, Q, tokens(new), N, d, O, ws[:least - 1])
