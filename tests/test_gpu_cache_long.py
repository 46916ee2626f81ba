"""Paged cache: one call whose units of work pass 2^31 (the division of the work is tested on the host in test_cache_ranges.py)."""
import math

import pytest
import torch

from paper_2603_17484_b200 import l2a

pytestmark = pytest.mark.gpu


def test_more_units_of_work_than_32_bits_count():
    """65536 routed tokens of 64 heads at the end of 2.2 million keys: 16384 groups of 256 rows, about 16900 key blocks each of 8 units."""
    Hq, Hkv, D, W, page, L, N = 64, 1, 64, 100, 128, 2_200_003, 65536
    assert N * Hq // 256 * (8 * ((L - N) // 128)) > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(1)
    n_pages = -(-L // page)
    K, V = (torch.randn((n_pages, Hkv, page, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "KV")
    table = torch.randperm(n_pages, generator=g, device="cuda").int()[None]
    handle = l2a.cache(K, V, table, torch.tensor([L], dtype=torch.int32, device="cuda"))
    Q = torch.randn((N, Hq, D), generator=g, device="cuda", dtype=torch.bfloat16)
    d = torch.ones(N, dtype=torch.uint8, device="cuda")
    O = torch.full_like(Q, float("nan"))
    p = l2a.params(1, N, L, Hq, Hkv, D, W)
    ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, handle, N), dtype=torch.uint8, device="cuda")
    l2a.l2a_cache_forward(p, handle, Q, None, N, d, O, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    assert bool(torch.isfinite(O).all())
    Kd, Vd = (x[table[0].long(), 0].reshape(-1, D)[:L].double() for x in (K, V))
    j = torch.arange(L, device="cuda")
    for t in (0, 1, 4097, 20000, 32767, 50001, N - 1):
        pos = L - N + t
        for h in (0, 37, 63):
            s = (Kd @ Q[t, h].double()) / math.sqrt(D)
            want, size = 0, 0
            for low in (pos - W, 0):
                x = torch.softmax(s[low:pos + 1], 0)
                want, size = want + x @ Vd[low:pos + 1], size + x @ Vd[low:pos + 1].abs()
            err = (O[t, h].double() - want).abs()
            # the bound of tests/cache_util.py
            assert bool((err <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -11) * size).all()), (t, h)
