"""Paged cache: sizes of the workspace around the decoded copy of an 8-bit cache (host only)."""
from paper_2603_17484_b200 import build as l2a_build
from paper_2603_17484_b200 import l2a
from tests.test_cache_host import WORKSPACE, cache, calls


def params(Lk):
    return l2a.params(16, 2000, Lk, 32, 8, 128, 4096)


def test_no_room_is_asked_for_a_copy_that_is_not_made():
    """A decoded copy beyond 4 GB is not made: the size is that of a bf16 cache."""
    l2a_build.build_lib()

    def size(Lk, kind):
        scales = dict(k_scale=None, v_scale=None) if kind == l2a.CACHE_BF16 else {}
        return l2a.l2a_cache_workspace_bytes(params(Lk), cache(table_stride=2048, kind=kind, **scales), 2000)
    assert size(131072, l2a.CACHE_E4M3) == size(131072, l2a.CACHE_BF16)                  # would be 8.6 GB
    assert size(32768, l2a.CACHE_E4M3) == size(32768, l2a.CACHE_BF16) + 4 * 16 * 32768 * 8 * 128
    # less than either is refused, before anything is launched
    c = cache(table_stride=2048)
    assert calls(params(131072), c, n=2000, ws_bytes=size(131072, l2a.CACHE_BF16) - 1)[2] == WORKSPACE
    assert calls(params(32768), c, n=2000, ws_bytes=size(32768, l2a.CACHE_BF16) - 1)[2] == WORKSPACE
