"""Eviction from a paged cache: refusals, all found on the host before any launch (no GPU is needed)."""
import ctypes

import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.test_cache_host import A, INVALID, UNSUPPORTED, WORKSPACE, cache, lib, params  # noqa: F401

OTHER = 0x40000


def evict(p=None, c=None, to=None, w=A, stride=0, keep=A, sinks=4, recent=8, w2=A, stride2=0, n2=A, kept=A, ws=A, ws_bytes=1 << 40):
    ref = ctypes.byref
    return l2a.lib().l2a_cache_evict(ref(p or params(Lq=100)), ref(c or cache()), w, stride, keep, sinks, recent,
                                     ref(to or cache(page_table=OTHER)), w2, stride2, n2, kept, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(w=None), INVALID), (dict(w2=None), INVALID), (dict(keep=None), INVALID), (dict(n2=None), INVALID), (dict(sinks=-1), INVALID),
    (dict(recent=-1), INVALID), (dict(w=A + 2), INVALID), (dict(w2=A + 1), INVALID), (dict(stride=2 * 64 - 1), INVALID),
    (dict(stride2=-1), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=A + 128), WORKSPACE), (dict(ws_bytes=0), WORKSPACE),
])
def test_arguments_that_are_refused(bad, code):
    assert evict(**bad) == code


@pytest.mark.parametrize("bad,code", [
    (dict(K=None), INVALID), (dict(k_scale=None), INVALID), (dict(page_size=24), UNSUPPORTED), (dict(kind=2), UNSUPPORTED),
    (dict(table_stride=0), INVALID), (dict(n_pages=0), INVALID),
])
def test_caches_that_are_refused(bad, code):
    assert evict(c=cache(**bad)) == code
    assert evict(to=cache(**{"page_table": OTHER, **bad})) == code
    with pytest.raises(l2a.L2AError) as e:
        l2a.l2a_cache_evict_workspace_bytes(params(Lq=100), cache(**bad))
    assert e.value.code == code


def test_caches_that_do_not_fit_each_other():
    assert evict(to=cache()) == INVALID                                          # the same pages
    assert evict(to=cache(page_table=OTHER, kind=l2a.CACHE_BF16, k_scale=None, v_scale=None)) == INVALID
    assert evict(to=cache(page_table=OTHER, table_stride=1)) == INVALID          # no room for what stays
    assert evict(p=params(Lq=100, D=96)) == UNSUPPORTED and evict(p=params(Lq=0)) == INVALID
    assert evict(p=params(Lq=100, B=70000)) == UNSUPPORTED


def test_workspace_is_enough_and_no_less():
    size = l2a.l2a_cache_evict_workspace_bytes(params(Lq=100), cache())
    assert evict(ws_bytes=size - 1) == WORKSPACE and size >= 2 * 2 * 100 * 4


def test_binding_refuses_weights_of_another_shape():
    K = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    c = l2a.cache(K, K, torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    good = torch.zeros((3, 2, 16))
    for w in (good.half(), good[:2], good.transpose(1, 2), torch.zeros((3, 2, 32))[:, :, ::2]):
        with pytest.raises(ValueError):
            l2a.l2a_cache_evict(l2a.params(1, 8, 48, 2, 2, 64, 0), c, w, None, 0, 0, c, good, None, None, None)
    assert l2a._weight_stride(torch.zeros((3, 4, 16))[:, :2], c) == 64
