"""4-bit caches: sequences of up to 64 rows are taken by the kernel of the few rows whatever the call's bounds, which shows in the rounding of the weights: fp16
there, bf16 in the chunks.  Values of one size and alternating signs: the result is small beside the sum of the weights, so that their rounding is what is seen.

Tolerance (tests/cache_util.py's, with fp16 weights): 2^-11 S for the weights, 2^-12 S for scores, exponentials and sums, one rounding of the result to bf16."""
import pytest
import torch

from tests.cache_e2m1_util import Cache4
from tests.cache_util import attention, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,new,lengths,Lk", [((32, 8, 128), 8, [12, 16, 30, 9], 200000), ((28, 4, 128), 9, [20, 11, 9], 400000),
                                                  ((16, 1, 64), 4, [70, 5, 6, 7, 8], 2000000)])
def test_weights_have_eleven_bits(heads, new, lengths, Lk):
    Hq, Hkv, D = heads
    sign = 1.0 - 2.0 * (torch.arange(max(lengths)) % 2)
    c = Cache4(128, Hkv, D, lengths, 3, per=-(-Lk // 128),
               rows=lambda which, b, x: x if which == 0 else sign[:len(x), None, None].expand_as(x).bfloat16())
    n = [new] * len(lengths)
    d = torch.zeros(sum(n), dtype=torch.uint8, device="cuda")
    for uniform in (False, True):
        O, Q = forward(c, Hq, n, 1000, d=d, Lk=Lk, uniform=uniform)
        o, size = attention(c, Q, n, d, 1000)
        err = (O.double() - o).abs()
        off = (2.0 ** -11 + 2.0 ** -12) * size
        assert bool((err <= off + 2.0 ** -8 * (o.abs() + off)).all()), float((err / size).max())
