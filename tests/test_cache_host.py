"""Paged cache: refusals, all found on the host before any launch (no GPU is needed), and the struct's layout."""
import ctypes

import pytest
import torch

from paper_2603_17484_b200 import build as l2a_build
from paper_2603_17484_b200 import l2a

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
A = 0x10000          # an address that nothing here follows


@pytest.fixture(scope="module", autouse=True)
def lib():
    l2a_build.build_lib()


def cache(**kw):
    f = dict(K=A, V=A, k_scale=A, v_scale=A, page_stride=0, scale_stride=0, kind=l2a.CACHE_E4M3, n_pages=10, page_size=64,
             table_stride=8, page_table=A, lengths=A)
    f.update(kw)
    return l2a.L2ACache(**f)


def params(**kw):
    f = dict(B=2, Lq=4, Lk=500, Hq=8, Hkv=2, D=128, window=16)
    f.update(kw)
    return l2a.params(**f)


def calls(p, c, n=8, cu=A, K=A, V=A, Q=A, O=A, ws=A, ws_bytes=1 << 40, d=A):
    """Codes of the three calls."""
    L, ref = l2a.lib(), ctypes.byref
    return (L.l2a_cache_append(ref(p), ref(c), K, V, cu, n, None), L.l2a_cache_read(ref(p), ref(c), None, K, V, None),
            L.l2a_cache_forward(ref(p), ref(c), Q, cu, n, d, O, ws, ws_bytes, None))


@pytest.mark.parametrize("bad,code", [
    (dict(K=0), INVALID), (dict(V=None), INVALID), (dict(page_table=None), INVALID), (dict(lengths=None), INVALID),
    (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(K=A + 8), INVALID), (dict(v_scale=A + 1), INVALID),
    (dict(kind=2), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
    (dict(page_size=256), UNSUPPORTED), (dict(n_pages=0), INVALID), (dict(table_stride=7), INVALID), (dict(table_stride=0), INVALID),
    (dict(page_stride=2 * 64 * 128 - 16), INVALID), (dict(page_stride=2 * 64 * 128 + 8), INVALID), (dict(scale_stride=120), INVALID),
    (dict(scale_stride=136), INVALID), (dict(page_stride=-16), INVALID),
])
def test_caches_that_are_refused(bad, code):
    assert calls(params(), cache(**bad)) == (code,) * 3
    with pytest.raises(l2a.L2AError) as e:
        l2a.l2a_cache_workspace_bytes(params(), cache(**bad), 8)
    assert e.value.code == code


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), INVALID), (dict(Lq=0), INVALID), (dict(Lk=0), INVALID), (dict(Hq=7), INVALID), (dict(D=80), UNSUPPORTED),
    (dict(window=-1), INVALID), (dict(softmax_scale=float("inf")), INVALID), (dict(softmax_scale=-1.0), INVALID),
    (dict(softmax_scale=float("nan")), INVALID), (dict(Lk=513), INVALID),
])
def test_parameters_that_are_refused(bad, code):
    assert calls(params(**bad), cache()) == (code,) * 3


def test_arguments_that_are_refused():
    p, c = params(), cache()
    assert calls(p, c, K=None)[:2] == (INVALID,) * 2 and calls(p, c, V=A + 2)[:2] == (INVALID,) * 2
    assert calls(p, c, n=-1)[0] == INVALID and calls(p, c, n=-1)[2] == INVALID
    for kw in (dict(Q=None), dict(O=None), dict(Q=A + 2), dict(O=A + 8)):
        assert calls(p, c, **kw)[2] == INVALID
    for kw in (dict(ws=None), dict(ws=A + 16), dict(ws_bytes=0), dict(ws_bytes=l2a.l2a_cache_workspace_bytes(p, c, 8) - 1)):
        assert calls(p, c, **kw)[2] == WORKSPACE
    # without cu_new every sequence has Lq new tokens
    assert calls(p, c, cu=None, n=7)[0] == INVALID and calls(p, c, cu=None, n=7)[2] == INVALID
    # strides of a token axis: no batch stride, whole 16 bytes, no overlap
    for s in ((64, 0), (0, 8 * 128 - 8), (0, 8 * 128 + 4), (0, -8)):
        assert calls(params(q_stride=s), c)[2] == INVALID and calls(params(o_stride=s), c)[2] == INVALID
    for s in ((64, 0), (0, 2 * 128 - 8), (0, 2 * 128 + 4)):
        assert calls(params(k_stride=s), c)[0] == INVALID and calls(params(v_stride=s), c)[0] == INVALID
    for s in ((499 * 256, 0), (0, 255), (-8, 0)):
        assert calls(params(k_stride=s), c)[1] == INVALID and calls(params(v_stride=s), c)[1] == INVALID


@pytest.mark.parametrize("flags,ok", [
    (0, True), (l2a.FLAG_SKIP_LOCAL, True), (l2a.FLAG_SKIP_GLOBAL, True), (l2a.FLAG_GLOBAL_PHASE, True),
    (l2a.FLAG_SHARED_WINDOW, True), (l2a.FLAG_SHARED_WINDOW | l2a.FLAG_SKIP_GLOBAL, True),
    (l2a.FLAG_SAVE_FOR_BWD, False), (l2a.FLAG_FORCE_ALL_GLOBAL, False), (l2a.FLAG_SKIP_LOCAL | l2a.FLAG_SKIP_GLOBAL, False),
    (l2a.FLAG_SKIP_LOCAL | l2a.FLAG_GLOBAL_PHASE, False), (1 << 30, False),
])
def test_flags(flags, ok):
    p = params(flags=flags)
    if ok:
        assert l2a.l2a_cache_workspace_bytes(p, cache(), 8) >= 256
    else:
        with pytest.raises(l2a.L2AError) as e:
            l2a.l2a_cache_workspace_bytes(p, cache(), 8)
        assert e.value.code == INVALID


def test_more_rows_than_32_bits_count():
    p, c = params(B=1, Lq=1 << 28, Lk=1 << 28), cache(table_stride=1 << 22)
    assert calls(p, c, n=1 << 28)[2] == UNSUPPORTED          # 2^31 rows


def test_no_tokens_are_no_work():
    """Nothing is launched for an empty token axis (this machine has no GPU to launch on)."""
    append, _, forward = calls(params(), cache(), n=0, K=None, V=None, Q=None, O=None)
    assert append == 0 and forward == 0


def test_workspace_grows_with_the_call():
    """The size for the largest call serves the smaller ones."""
    for heads in ((28, 4, 128), (12, 2, 64), (8, 1, 128)):
        def size(B, Lq, Lk, n, **kw):
            return l2a.l2a_cache_workspace_bytes(l2a.params(B, Lq, Lk, *heads, 128), cache(table_stride=4096, **kw), n)
        most = size(8, 500, 100000, 4000)
        for n in (1, 7, 8, 64, 500, 3999):
            for Lq in (1, 3, 17, 499):
                for Lk in (1, 64, 5000, 100000):
                    assert 256 <= size(8, Lq, Lk, n) <= most, (n, Lq, Lk)


def test_struct_layout_matches_header():
    # four pointers, two 64-bit strides, four 32-bit fields, two pointers
    assert ctypes.sizeof(l2a.L2ACache) == 4 * 8 + 2 * 8 + 4 * 4 + 2 * 8
    assert l2a.L2ACache.kind.offset == 48 and l2a.L2ACache.page_table.offset == 64


def test_binding_refuses_mixed_tensors():
    K = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    q = torch.zeros((3, 2, 16, 64), dtype=torch.uint8)
    e = torch.zeros((3, 2, 16), dtype=torch.uint8)
    table, n = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    assert l2a.cache(K, K, table, n).kind == l2a.CACHE_BF16
    c = l2a.cache(q, q, table, n, e, e)
    assert (c.kind, c.n_pages, c.page_size, c.page_stride) == (l2a.CACHE_E4M3, 3, 16, 2 * 16 * 64)
    for args in ((K, q, table, n), (K, K, table, n, e, e), (q, q, table, n), (q, q, table, n, e, None), (q, q, table, n, e[:2], e[:2]),
                 (K, K[:2], table, n), (K, K, table.long(), n), (K, K, table, n.long()), (K.float(), K.float(), table, n),
                 (K.transpose(2, 3), K.transpose(2, 3), table, n)):
        with pytest.raises(ValueError):
            l2a.cache(*args)
