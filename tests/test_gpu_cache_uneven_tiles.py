"""Paged cache, chunks: the two tiles of a group of rows have their key blocks far apart.  The routed tokens are the first ones of the
chunk and a few at its end, so that the first tile is done many blocks before the second and goes on to the CTA's next piece; the sizes
of the values differ from block to block, so that a scale of another block would show."""
import pytest
import torch

from tests.cache_util import Cache, attention, check, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,B,new,last", [((16, 16, 64), 3, 1500, 40), ((16, 16, 64), 2, 1300, 128), ((6, 6, 128), 6, 1400, 3),
                                              ((4, 2, 64), 8, 760, 20)])
def test_tiles_far_apart(kind, heads, B, new, last):
    Hq, Hkv, D = heads
    L, W = new + 300, 64
    g = torch.Generator().manual_seed(new)
    size = 2.0 ** torch.randint(-5, 6, (-(-L // 32),), generator=g).double().repeat_interleave(32)[:L, None, None]
    c = Cache(kind, 64, Hkv, D, [L] * B, 17, v_scale=size)
    first = 128 * Hkv // Hq
    d = torch.zeros((B, new), dtype=torch.uint8)
    d[:, :first] = 1
    d[:, new - last:] = 1
    d = d.flatten().cuda()
    O, Q = forward(c, Hq, [new] * B, W, d=d, seed=3)
    want, bound = attention(c, Q, [new] * B, d, W)
    check(O, want, bound, f"{kind} {heads} {new} new, {first} and {last} routed")
