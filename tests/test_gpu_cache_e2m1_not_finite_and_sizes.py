"""4-bit caches: NaN in a query row stays with that row, on every path; values and keys of very unequal size.  Definition and tolerance:
tests/cache_util.py, tests/cache_e2m1_util.py."""
import pytest
import torch

from tests.cache_e2m1_util import Cache4
from tests.cache_util import Cache, attention, check, forward, routed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("heads,lengths,new,W", [
    ((28, 4, 128), [60, 40], [1, 1], 100),               # one piece a sequence
    ((28, 4, 128), [9000, 700], [1, 1], 100),            # parts that are combined
    ((8, 1, 64), [9000, 700], [3, 2], 100),              # blocks of 16 rows
    ((28, 4, 128), [700, 300], [40, 40], 100),           # chunks
    ((32, 8, 128), [3000], [600], 100),                  # from a decoded copy
])
def test_a_query_row_that_is_not_finite(heads, lengths, new, W, value):
    Hq, Hkv, D = heads
    c = Cache4(64, Hkv, D, lengths, 28)
    N = sum(new)
    d = routed(N, 0.5, 3)
    d[0], d[N - 1] = 1, 0
    Q = torch.randn((N, Hq, D), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    want, size = attention(c, Q, new, d, W)
    bad = torch.zeros((N, Hq), dtype=torch.bool, device="cuda")
    for t, h, e in ((0, 1, 3), (N - 1, Hq - 1, D - 1), (N // 2, 0, 0)):
        Q[t, h, e] = value
        bad[t, h] = True
    O = forward(c, Hq, new, W, d=d, Q=Q)[0]
    if value != value:
        assert bool(O[bad].isnan().all())
    check(O[~bad], want[~bad], size[~bad], f"{heads} {new}")


@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 1, 64)])
@pytest.mark.parametrize("size", [1e-6, 1e-10, 1e-30])
@pytest.mark.parametrize("new", [1, 5, 40, 230])
def test_zero_rows_among_small_values(heads, size, new):
    Hq, Hkv, D = heads
    L = 500
    for every in (5, 1):
        x = torch.full((L, 1, 1), size, dtype=torch.float64)
        x[::every] = 0.0
        c = Cache4(32, Hkv, D, [L, L], 23, v_scale=x)
        d = routed(2 * new, 0.6, new)
        O, Q = forward(c, Hq, [new] * 2, 100, d=d, seed=2)
        check(O, *attention(c, Q, [new] * 2, d, 100), f"{heads} values {size}, zeros every {every}")


@pytest.mark.parametrize("new", [1, 5, 9, 40, 300])
@pytest.mark.parametrize("size", [2.0 ** 22, 1e15, 1e30])
def test_values_of_later_tokens(new, size):
    """The values of the last two tokens are `size` times the others': nothing of that reaches the rows before them.

    Few rows: a weight is fp16 at a scale at which the largest P_j 2^e_j that the row sees is 2^10 at least, so that it is off by 2^-25 at most besides its 11
    bits, 2^-35 of that largest; a value is 2^e times 2688 at most and its row's largest, v_j, above 2^e times 1344.  A column whose
    codes of the large tokens are zeros sees that: n keys are off by n 2^-35 2688 max P_j 2^e_j <= n 2^-34 max P_j v_j <= n 2^-34 sum P_j v_j together."""
    L, Hq, Hkv, D, W = 600, 28, 4, 128, 60
    x = torch.full((L, 1, 1), 1e-5, dtype=torch.float64)
    x[-2:] *= size
    c = Cache4(64, Hkv, D, [L, L], 24, v_scale=x)
    d = routed(2 * new, 0.6, new)
    O, Q = forward(c, Hq, [new] * 2, W, d=d, seed=2)
    want, bound = attention(c, Q, [new] * 2, d, W)
    if new * Hq // Hkv <= 64:
        V = c.V
        c.V = [v.abs().amax(-1, keepdim=True).expand_as(v) for v in V]
        least = L * 2.0 ** -34 * attention(c, Q, [new] * 2, d, W)[1]
        O = torch.where((O.double() - want).abs() <= least, want, O.double())            # (what is within that of the result counts as the result)
    check(O, want, bound, f"new {new} size {size}")


@pytest.mark.parametrize("new", [1, 2, 9, 40, 300])
@pytest.mark.parametrize("step", [1.0, 30.0, -30.0])
def test_scores_that_grow_and_fall_along_the_keys(new, step):
    """Each 64 keys' scores are `step` binary orders above the last ones': the reference of a row has to follow, or to stay."""
    L, Hq, Hkv, D = 900, 8, 2, 128
    q = torch.ones((2 * new, Hq, D)).bfloat16().cuda()
    level = (torch.arange(L) // 64).double() * step * 0.7 / D * D ** 0.5

    def rows(which, b, x):
        return (level[:, None, None].expand_as(x).clone() + 0.05 * x.double()).bfloat16() if which == 0 else x
    c = Cache4(32, Hkv, D, [L, L], 5, rows=rows)
    d = routed(2 * new, 0.6, new)
    O, Q = forward(c, Hq, [new] * 2, 400, d=d, Q=q)
    check(O, *attention(c, Q, [new] * 2, d, 400), f"new {new} step {step}")


@pytest.mark.parametrize("heads,lengths,new", [((28, 4, 128), [700, 300], [30, 40]), ((28, 4, 128), [700, 300], [230, 40]), ((8, 1, 64), [900], [100])])
def test_chunks_equal_those_from_what_the_codes_stand_for(heads, lengths, new):
    """The same bits as from a bf16 cache of the decoded values: elements of Q of every size, an infinite one."""
    Hq, Hkv, D = heads
    c, b = Cache4(64, Hkv, D, lengths, 26), Cache("bf16", 64, Hkv, D, lengths, 26)
    for i, n in enumerate(lengths):
        j = torch.arange(n, device="cuda")
        pages = b.table[i].long()[j // 64]
        b.poolK[pages, :, j % 64] = c.K[i].bfloat16()
        b.poolV[pages, :, j % 64] = c.V[i].bfloat16()
    N = sum(new)
    g = torch.Generator().manual_seed(4)
    Q = torch.randn((N, Hq, D), generator=g) * 2.0 ** torch.randint(-30, 3, (N, Hq, D), generator=g)
    Q[3, 1, 7] = float("inf")
    Q = Q.bfloat16().cuda()
    d = routed(N, 0.6, 1)
    x, y = (forward(k, Hq, new, 100, d=d, Q=Q)[0] for k in (c, b))
    assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x.nan_to_num(), y.nan_to_num())
    assert bool(x[3, 1].isnan().any()) and not bool(x[0].isnan().any())
