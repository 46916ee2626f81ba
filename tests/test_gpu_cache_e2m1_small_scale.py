"""4-bit caches, few rows: soft-max scales so small that they leave fp32 together with the power of two that brings a row of queries to fp16's range.  The
weights are then all but equal: the attention is the mean of the values that a row sees, the weight of a key the sum of 1 / (keys seen)."""
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache
from tests.cache_util import attention, check, forward
from tests.cache_weigh_util import weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["e2m1", "e4m3", "bf16"])
@pytest.mark.parametrize("q_size", [0.0, 1e-38, 1.0])
@pytest.mark.parametrize("scale", [1e-20, 1e-38])
@pytest.mark.parametrize("new", [[1, 1], [5, 2]])
def test_attention(kind, q_size, scale, new):
    c = make_cache(kind, 64, 2, 128, [700, 90], 9)
    Q = (torch.randn((sum(new), 8, 128), generator=torch.Generator().manual_seed(1)).double() * q_size).bfloat16().cuda()
    d = torch.tensor([1] + [0] * (sum(new) - 2) + [1], dtype=torch.uint8).cuda()
    O, _ = forward(c, 8, new, 100, d=d, Q=Q, scale=scale)
    check(O, *attention(c, Q, new, d, 100, scale=scale), f"{kind} {q_size} {scale}")


@pytest.mark.parametrize("kind", ["e2m1", "e4m3", "bf16"])
@pytest.mark.parametrize("q_size", [0.0, 1e-38])
def test_weights(kind, q_size):
    c, new, scale = make_cache(kind, 64, 2, 128, [700, 90], 9), [3, 2], 1e-20
    Q = (torch.randn((5, 8, 128), generator=torch.Generator().manual_seed(1)).double() * q_size).bfloat16().cuda()
    w = torch.zeros((c.poolK.shape[0], 2, 64), device="cuda")
    p = l2a.params(2, 3, 700, 8, 2, 128, 0, softmax_scale=scale)
    ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, 5), dtype=torch.uint8, device="cuda")
    l2a.l2a_cache_weigh(p, c.handle, Q, torch.tensor([0, 3, 5], dtype=torch.int32).cuda(), 5, None, w, ws)
    for b, (inc, off) in enumerate(weights(c, Q, new, torch.ones(5, device="cuda"), scale)):
        j = torch.arange(c.lengths[b], device="cuda")
        got = w[c.table[b, j // 64].long(), :, j % 64].double()
        assert bool(((got - inc).abs() <= off + 2.0 ** -24 * inc).all())
