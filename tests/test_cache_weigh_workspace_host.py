"""Weights of cached keys: a workspace that is sized once for the largest step is enough for every smaller one (host only)."""
import pytest

from paper_2603_17484_b200 import l2a
from tests.test_cache_host import cache, lib  # noqa: F401
from tests.test_cache_weigh_host import weigh

KINDS = [l2a.CACHE_BF16, l2a.CACHE_E4M3, l2a.CACHE_E2M1]


def case(B, Lq, Lk, heads, kind):
    scales = dict(k_scale=None, v_scale=None) if kind == l2a.CACHE_BF16 else {}
    return l2a.params(B, Lq, Lk, *heads, 0), cache(kind=kind, table_stride=1 << 14, **scales)


def size(B, Lq, Lk, heads, kind, n):
    return l2a.l2a_cache_weigh_workspace_bytes(*case(B, Lq, Lk, heads, kind), n)


# around the bound of the scores, 4 GB: rows of scores are kept or not as tokens and keys grow
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,heads", [(22, (32, 8, 128)), (64, (24, 1, 128)), (1, (28, 4, 128)), (300, (8, 8, 64)), (7, (80, 1, 64)), (1000, (12, 2, 64))])
def test_size_grows_with_tokens_and_keys(B, heads, kind):
    keys = [1, 64, 1000, 9000, 32768, 50000, 65000, 100000, 131072, 300000, 600000]
    tokens = [1, 2, 3, 4, 5, 7, 8, 11, 12, 15, 16, 17, 24, 33, 64, 65, 500, 2000]
    got = [[size(B, Lq, Lk, heads, kind, B) for Lq in tokens] for Lk in keys]
    for i, row in enumerate(got):
        assert all(x <= y for x, y in zip(row, row[1:])), f"{keys[i]} keys: {row}"
    for j in range(len(tokens)):
        column = [row[j] for row in got]
        assert all(x <= y for x, y in zip(column, column[1:])), f"{tokens[j]} tokens: {column}"


@pytest.mark.parametrize("kind", KINDS)
def test_a_smaller_step_is_taken(kind):
    """A server's workspace for chunks of 500, then steps of a few tokens of shorter sequences.  (No tokens: nothing is launched.)"""
    heads = (32, 8, 128)
    large = size(22, 500, 131072, heads, kind, 2000)
    for Lq, Lk in ((11, 131072), (8, 100000), (16, 90000), (1, 131072), (500, 60000)):
        p, c = case(22, Lq, Lk, heads, kind)
        assert weigh(p=p, c=c, n=0, Q=None, w=None, ws_bytes=large) == 0
        assert size(22, Lq, Lk, heads, kind, min(22 * Lq, 2000)) <= large


def test_without_the_bound_the_size_is_that_of_the_call():
    """Where all scores fit, what a smaller step needs does not add to the size: 64 rows of 32768 keys, 8 heads, and little else."""
    n = size(4, 16, 32768, (32, 8, 128), l2a.CACHE_E2M1, 64)
    assert 4 * 4 * 8 * 64 * 32768 <= n <= 4 * 4 * 8 * 64 * 32768 + (1 << 20)
