"""Weights of cached keys: refusals, all found on the host before any launch (no GPU is needed), and the workspace."""
import ctypes

import pytest

from paper_2603_17484_b200 import l2a
from tests.test_cache_host import A, INVALID, UNSUPPORTED, WORKSPACE, cache, lib, params  # noqa: F401


def weigh(p=None, c=None, Q=A, cu=A, n=8, d=A, w=A, stride=0, ws=A, ws_bytes=1 << 50):
    ref = ctypes.byref
    return l2a.lib().l2a_cache_weigh(ref(p or params()), ref(c or cache()), Q, cu, n, d, w, stride, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(Q=None), INVALID), (dict(Q=A + 8), INVALID), (dict(w=None), INVALID), (dict(w=A + 2), INVALID), (dict(stride=2 * 64 - 1), INVALID),
    (dict(stride=-1), INVALID), (dict(n=-1), INVALID), (dict(cu=None, n=7), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=A + 8), WORKSPACE),
    (dict(ws_bytes=0), WORKSPACE), (dict(c=cache(K=None)), INVALID), (dict(c=cache(kind=2)), UNSUPPORTED), (dict(c=cache(lengths=None)), INVALID),
    (dict(p=params(D=96)), UNSUPPORTED), (dict(p=params(Hq=7)), INVALID), (dict(p=params(q_stride=(0, 8 * 128 - 8))), INVALID),
    (dict(p=params(q_stride=(64, 0))), INVALID), (dict(p=params(softmax_scale=-1.0)), INVALID), (dict(p=params(B=70000)), UNSUPPORTED),
    (dict(p=params(flags=l2a.FLAG_SKIP_LOCAL)), INVALID), (dict(p=params(flags=l2a.FLAG_GLOBAL_PHASE)), INVALID),
])
def test_refusals(bad, code):
    assert weigh(**bad) == code


def test_no_tokens_are_no_work():
    assert weigh(n=0, Q=None, w=None) == 0


def test_more_rows_than_32_bits_count():
    assert weigh(p=params(B=1, Lq=1 << 28, Lk=1 << 28), c=cache(table_stride=1 << 22), n=1 << 28) == UNSUPPORTED


def test_workspace():
    def size(B, Lq, Lk, n, heads=(32, 8, 128), kind=l2a.CACHE_E2M1):
        return l2a.l2a_cache_weigh_workspace_bytes(l2a.params(B, Lq, Lk, *heads, 0), cache(kind=kind, table_stride=1 << 14), n)
    p, c = params(), cache()
    need = l2a.l2a_cache_weigh_workspace_bytes(p, c, 8)
    assert weigh(ws_bytes=need - 1) == WORKSPACE
    # scores of 4 rows of 8 heads
    assert 4 * 16 * 8 * 4 * 32768 <= size(16, 1, 32768, 16) < 4.2 * 16 * 8 * 4 * 32768
    # never more than 4 GB of them, whatever the batch
    assert size(1000, 16, 100000, 1000, kind=l2a.CACHE_BF16) < 5 << 30
    for n in (1, 7, 64, 1999):
        assert size(4, 500, 9000, n) <= size(4, 500, 9000, 2000)
    # many rows of codes: the keys in bf16
    assert size(1, 1000, 20000, 1000) - size(1, 1000, 20000, 1000, kind=l2a.CACHE_BF16) >= 2 * 20000 * 8 * 128
