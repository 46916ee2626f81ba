"""Paged cache: values of very unequal size.  Rows of zeros (exponent 0 in the 8-bit format) among small values must not cost the others
their bits.  Tolerance and definition: tests/cache_util.py."""
import pytest
import torch

from tests.cache_util import Cache, attention, check, forward, routed

pytestmark = pytest.mark.gpu


def zeros_among(L, size, every):
    x = torch.full((L, 1, 1), size, dtype=torch.float64)
    x[::every] = 0.0
    return x


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 1, 64)])
@pytest.mark.parametrize("size", [1e-6, 1e-10, 1e-30])
@pytest.mark.parametrize("new", [1, 5])
def test_zero_rows_among_small_values(kind, heads, size, new):
    """Every fifth value row is zeros, inside the window and before it; then all of them."""
    Hq, Hkv, D = heads
    L = 500
    for every in (5, 1):
        c = Cache(kind, 32, Hkv, D, [L, L], 23, v_scale=zeros_among(L, size, every))
        d = routed(2 * new, 0.6, new)
        O, Q = forward(c, Hq, [new] * 2, 100, d=d, seed=2)
        want, bound = attention(c, Q, [new] * 2, d, 100)
        check(O, want, bound, f"{kind} {heads} values {size}, zeros every {every}")
