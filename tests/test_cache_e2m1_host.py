"""4-bit paged caches: refusals found on the host, the binding, and properties of the format (no GPU is needed)."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import decoded4, quantise4
from tests.test_cache_host import A, INVALID, UNSUPPORTED, cache, calls, lib, params  # noqa: F401


def cache4(**kw):
    return cache(**{"kind": l2a.CACHE_E2M1, **kw})


@pytest.mark.parametrize("bad,code", [
    (dict(K=0), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(V=A + 8), INVALID), (dict(k_scale=A + 8), INVALID),
    (dict(page_size=8), UNSUPPORTED), (dict(page_stride=2 * 64 * 128 - 32), INVALID), (dict(page_stride=2 * 64 * 128 + 16), INVALID),
    (dict(scale_stride=2 * 64 * 9 - 16), INVALID), (dict(scale_stride=2 * 64 * 9 + 8), INVALID), (dict(scale_stride=2 * 64), INVALID),
    (dict(page_stride=1 << 62), INVALID),
])
def test_caches_that_are_refused(bad, code):
    assert calls(params(), cache4(**bad)) == (code,) * 3


def test_strides_that_are_taken():
    p = params()
    for ok in (dict(), dict(page_stride=2 * 64 * 128 + 32), dict(scale_stride=2 * 64 * 9 + 16)):
        assert l2a.l2a_cache_workspace_bytes(p, cache4(**ok), 8) >= 256


def test_workspace_of_a_decoded_copy():
    """Many rows: the same workspace as for 8 bits; few: none of the kinds needs a copy."""
    for Lq in (1, 8, 1000):
        p = params(Lq=Lq, Lk=8000)
        size = [l2a.l2a_cache_workspace_bytes(p, cache(kind=k, table_stride=200), 2 * Lq) for k in (l2a.CACHE_BF16, l2a.CACHE_E4M3, l2a.CACHE_E2M1)]
        assert size[0] <= size[2] and size[1] <= size[2]


def test_binding():
    table, n = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    K = torch.zeros((3, 2, 16, 32), dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    e = torch.zeros((3, 2, 16 * 5), dtype=torch.uint8)
    c = l2a.cache(K, K, table, n, e, e)
    assert (c.kind, c.n_pages, c.page_size, c.page_stride, c.scale_stride) == (l2a.CACHE_E2M1, 3, 16, 2 * 16 * 64, 2 * 16 * 5)
    apart = torch.zeros((3, 2, 2, 16, 32), dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    assert l2a.cache(apart[:, 0], apart[:, 1], table, n, e, e).page_stride == 2 * 2 * 16 * 64
    u8 = torch.zeros((3, 2, 16, 32), dtype=torch.uint8)
    for args in ((K, u8, table, n, e, e), (K, K, table, n), (K, K, table, n, e, None), (K, K, table, n, e[:, :, :16], e[:, :, :16]),
                 (K, K, table, n, e.char(), e.char()), (K, K, table, n, e[:2], e[:2]), (K, K[:2], table, n, e, e)):
        with pytest.raises(ValueError):
            l2a.cache(*args)


def test_error_of_the_format():
    """A value is off by at most a sixth of its block's scale times six (half the widest step of e2m1, 1), a rounding of the scale
    (2^-4) that takes the largest values beyond 6 among it, and half the least step of the scales."""
    r = np.random.default_rng(3)
    x = (r.standard_normal((4000, 128)) * np.exp(2 * r.standard_normal((4000, 1)))).astype(np.float32)
    x = torch.from_numpy(x).bfloat16().double().numpy()
    q, s, e = quantise4(x)
    y = decoded4(q, s, e)
    top = np.abs(x).reshape(4000, 8, 16).max(-1).repeat(16, -1)
    assert (np.abs(y - x) <= top / 6 * (1 + 2.0 ** -4) + top * 2.0 ** -4 + 6 * 2.0 ** -10 * np.exp2(e - 127.0)[:, None]).all()
    assert np.array_equal(torch.from_numpy(y).bfloat16().double().numpy(), y)          # exact in bf16
