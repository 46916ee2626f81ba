"""Paged cache: more new tokens than the sequence is long.  Rows at positions below 0 see nothing and get zeros; the others are those of the
definition, in both kinds of caches, on every path (tests/cache_util.py has the tolerance)."""
import pytest
import torch

from tests.cache_util import Cache, attention, check, forward, routed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads", [(28, 4, 128), (4, 4, 64), (32, 8, 128)])
@pytest.mark.parametrize("lengths,new", [([2, 5], [4, 1]), ([3, 1], [2, 2]), ([30, 40], [60, 20]), ([200, 3, 90], [300, 40, 90]),
                                         ([500, 20], [400, 30])])
def test_rows_ahead_of_the_first_position(kind, heads, lengths, new):
    Hq, Hkv, D = heads
    for W, density in ((8, 1.0), (50, 0.5)):
        c = Cache(kind, 16, Hkv, D, lengths, 30, per=32)
        d = routed(sum(new), density, 3)
        O, Q = forward(c, Hq, new, W, d=d, Lk=512)
        want, size = attention(c, Q, new, d, W)
        check(O, want, size, f"{kind} {heads} {lengths} new {new} W {W}")
        t = 0
        for length, n in zip(lengths, new):
            assert not O[t:t + max(0, n - length)].any()
            t += n


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("new", [[1, 2], [3, 5], [70, 1], [300, 20]])
def test_sequences_without_a_token(kind, new):
    """Lengths of zero, beside one that has tokens."""
    c = Cache(kind, 32, 4, 128, [40, 40], 31, per=16)
    c.length.copy_(torch.tensor([0, 40]))
    d = torch.ones(sum(new), dtype=torch.uint8, device="cuda")
    O, Q = forward(c, 28, new, 8, d=d, Lk=512)
    assert not O[:new[0]].any()
    c.lengths, c.K, c.V = [40], c.K[1:], c.V[1:]
    want, size = attention(c, Q[new[0]:], new[1:], d[new[0]:], 8)
    check(O[new[0]:], want, size, f"{kind} {new}")
