"""Paged cache, few rows: the workspace holds a part for each pair of a sequence and KV head and for each CTA that the cache's kind has, no more
(host only).  A workspace of a fixed size that was enough for 16- and 8-bit caches stays enough."""
import pytest

from paper_2603_17484_b200 import l2a
from tests.test_cache_host import cache, lib  # noqa: F401

SMS = 148


def up(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("kind,per_sm", [(l2a.CACHE_BF16, 2), (l2a.CACHE_E4M3, 2), (l2a.CACHE_E2M1, 3)])
@pytest.mark.parametrize("B,Lq,heads", [(1, 1, (28, 4, 128)), (16, 1, (32, 8, 128)), (70, 2, (32, 8, 64)), (3, 1, (12, 1, 64)), (5, 2, (16, 2, 128))])
def test_a_part_for_each_cta(kind, per_sm, B, Lq, heads):
    Hq, Hkv, D = heads
    rows = Lq * Hq // Hkv
    assert rows <= 16
    if rows > 8:
        per_sm = 2
    scales = dict(k_scale=None, v_scale=None) if kind == l2a.CACHE_BF16 else {}
    got = l2a.l2a_cache_workspace_bytes(l2a.params(B, Lq, 9000, *heads, 100), cache(kind=kind, table_stride=1 << 10, **scales), B * Lq)
    parts = (2 * B * Hkv + per_sm * SMS) * (16 if rows > 8 else 8) * (D + 4) * 4
    assert got == 256 + up((B + 1) * 32) + up(parts)
