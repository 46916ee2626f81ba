"""Calls at the edges of what 4-bit caches, weights of cached keys and evictions allow: every quotient of the format, lists that end before the
last row, sequences shorter than their new tokens, bounds above what there is, calls on two streams at once."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache, quantise4
from tests.cache_util import attention, check, routed
from tests.cache_weigh_util import weights

pytestmark = pytest.mark.gpu


def every_quotient(D):
    """Rows whose first value, 2688, makes the exponent 0.  Each other block has one of all bf16 from 2^-12 (below the least scale) to 2688 as its
    largest, the rest are values of all mantissas of the seven powers of two below it."""
    bf16 = np.ldexp(1 + np.arange(128) / 128, np.arange(-12, 12)[:, None]).reshape(-1)
    bf16 = bf16[bf16 <= 2688]
    below = np.ldexp(1 + np.arange(128) / 128, -np.arange(7)[:, None]).reshape(-1)
    below = np.concatenate([below, np.zeros(-len(below) % 15)]).reshape(-1, 15)
    power = np.exp2(np.floor(np.log2(bf16)))
    blocks = np.empty((len(bf16), len(below), 16))
    blocks[..., 0] = bf16[:, None]
    blocks[..., 1:] = np.minimum(below * power[:, None, None], bf16[:, None, None])
    blocks[..., 1::2] *= -1
    blocks = blocks.reshape(-1, 16)
    per = D // 16 - 1
    blocks = np.concatenate([blocks, np.zeros((-len(blocks) % per, 16))]).reshape(-1, per * 16)
    first = np.zeros((len(blocks), 16))
    first[:, 0] = 2688
    return np.concatenate([first, blocks], 1)


@pytest.mark.parametrize("D", [64, 128])
def test_every_quotient_is_rounded_as_the_format_says(D):
    rows = every_quotient(D)
    N = len(rows)
    x = torch.from_numpy(rows).bfloat16()
    assert torch.equal(x.double(), torch.from_numpy(rows))
    pages = -(-N // 128)
    codes = torch.zeros((2, pages, 1, 128, D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((2, pages, 1, 128 * (1 + D // 16)), dtype=torch.uint8, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    four = torch.float4_e2m1fn_x2
    c = l2a.cache(codes[0].view(four), codes[1].view(four), table, torch.tensor([N], dtype=torch.int32, device="cuda"), k_scale=scales[0], v_scale=scales[1])
    x = x.cuda()[:, None]
    l2a.l2a_cache_append(l2a.params(1, N, N, 1, 1, D, 0), c, x, -x, None, N)
    torch.cuda.synchronize()
    for which, sign in ((0, 1.0), (1, -1.0)):
        q, s, e = quantise4(sign * rows)
        got = scales[which].cpu().numpy()[:, 0]
        assert np.array_equal(got[:, :128].reshape(-1)[:N], e)
        assert np.array_equal(got[:, 128:].reshape(-1, D // 16)[:N], s)
        assert np.array_equal(codes[which].cpu().numpy().reshape(-1, D // 2)[:N], q)


def odd_call(kind, lengths, new, Hq, Hkv, D, page, seed):
    """A call's cache, bounds, list and inputs: rows behind the last sequence, bounds above what there is."""
    Lk = max(lengths) + 200
    c = make_cache(kind, page, Hkv, D, lengths, seed, per=-(-Lk // page))
    N = sum(new)
    g = torch.Generator().manual_seed(seed)
    Q = torch.randn((N + 5, Hq, D), generator=g).bfloat16().cuda()
    d = routed(N + 5, 0.5, seed)
    d[N - 1:] = 1
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    p = l2a.params(len(new), max(new) + 7, Lk, Hq, Hkv, D, 60)
    return c, Q, d, cu, p, N


ODD = [([300, 0, 2, 150], [1, 1, 3, 2]), ([500, 0, 100, 3, 40], [40, 2, 130, 9, 0]), ([1000, 200, 90], [200, 300, 1])]


@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 2, 64)])
@pytest.mark.parametrize("lengths,new", ODD)
def test_attention_of_odd_calls(lengths, new, heads):
    c, Q, d, cu, p, N = odd_call("e2m1", lengths, new, *heads, 32, 5)
    O = torch.full_like(Q, 7.0)
    ws = torch.full((l2a.l2a_cache_workspace_bytes(p, c.handle, len(Q)),), 0xA5, dtype=torch.uint8, device="cuda")
    l2a.l2a_cache_forward(p, c.handle, Q, cu, len(Q), d, O, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    assert bool((O[N:] == 7).all())
    t = 0
    for b, n in enumerate(new):
        got, t = O[t:t + n], t + n
        if lengths[b] == 0:
            assert not got.any()
        elif n:
            one = SimpleNamespace(K=c.K[b:b + 1], V=c.V[b:b + 1], lengths=lengths[b:b + 1], Hkv=c.Hkv)
            want, size = attention(one, Q[t - n:t], [n], d[t - n:t], 60)
            check(got, want, size, f"{lengths} {new}: sequence {b}")


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("lengths,new", ODD)
def test_weights_of_odd_calls(kind, lengths, new):
    c, Q, d, cu, p, N = odd_call(kind, lengths, new, 28, 4, 128, 32, 6)
    pool = torch.rand((c.poolK.shape[0], 4, 32), generator=torch.Generator().manual_seed(1)).cuda()
    before = pool.clone()
    ws = torch.full((l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, len(Q)),), 0xA5, dtype=torch.uint8, device="cuda")
    l2a.l2a_cache_weigh(p, c.handle, Q, cu, len(Q), d, pool, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    rest = torch.ones_like(pool, dtype=torch.bool)
    t = 0
    for b, (inc, off) in enumerate(weights(c, Q[:N], new, d[:N])):
        n, length = new[b], lengths[b]
        j = torch.arange(length, device="cuda")
        at, slot = c.table[b, j // 32].long(), j % 32
        old = before[at, :, slot].double()
        old[max(length - n, 0):] = 0
        want = old + inc if n else before[at, :, slot].double()
        rows = int(d[t:t + n].sum()) * 7
        bound = off + max(1, -(-rows // 512)) * 2.0 ** -24 * want + 1e-36
        assert bool(((pool[at, :, slot].double() - want).abs() <= bound).all()), f"sequence {b}"
        rest[at, :, slot] = False
        t += n
    assert torch.equal(pool[rest], before[rest])


def test_calls_on_two_streams_at_once_give_the_bits_of_each_alone():
    Hq, Hkv, D = 28, 4, 128
    calls = []
    for k, (lengths, new) in enumerate((([3000, 2500], [1, 1]), ([2000, 900], [300, 80]))):
        c = make_cache("e2m1", 64, Hkv, D, lengths, k)
        N = sum(new)
        p = l2a.params(2, max(new), max(lengths), Hq, Hkv, D, 500)
        cu = torch.tensor([0, new[0], N], dtype=torch.int32).cuda()
        Q, d = torch.randn((N, Hq, D), device="cuda").bfloat16(), routed(N, 0.5, k)
        d[0] = 1
        ws = [torch.empty(f(p, c.handle, N), dtype=torch.uint8, device="cuda") for f in (l2a.l2a_cache_workspace_bytes, l2a.l2a_cache_weigh_workspace_bytes)]
        O, w = torch.zeros_like(Q), torch.zeros((c.poolK.shape[0], Hkv, 64), device="cuda")
        to = make_cache("e2m1", 32, Hkv, D, [1000, 1000], k)
        w2, n2 = torch.zeros((to.poolK.shape[0], Hkv, 32), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        keep = torch.tensor([700, 800], dtype=torch.int32, device="cuda")
        pe = l2a.params(2, 1000, max(lengths), Hkv, Hkv, D, 0)
        wse = torch.empty(l2a.l2a_cache_evict_workspace_bytes(pe, c.handle), dtype=torch.uint8, device="cuda")

        def run(c=c, p=p, cu=cu, Q=Q, d=d, ws=ws, O=O, w=w, to=to, w2=w2, n2=n2, keep=keep, pe=pe, wse=wse, N=N):
            l2a.l2a_cache_forward(p, c.handle, Q, cu, N, d, O, ws[0])
            l2a.l2a_cache_weigh(p, c.handle, Q, cu, N, d, w, ws[1])
            l2a.l2a_cache_evict(pe, c.handle, w, keep, 4, 500, to.handle, w2, n2, None, wse)
        calls.append((run, [O, w, to.codes, to.scales, w2, n2]))
    alone = []
    for run, out in calls:
        run()
        torch.cuda.synchronize()
        alone.append([x.clone() for x in out])
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for (_, out) in calls:
            out[1].zero_()
        torch.cuda.synchronize()
        for (run, _), s in zip(calls, streams):
            with torch.cuda.stream(s):
                run()
        torch.cuda.synchronize()
        for (_, out), want in zip(calls, alone):
            for a, b in zip(out, want):
                assert torch.equal(a.view(torch.uint8) if a.dtype != torch.int32 else a, b.view(torch.uint8) if b.dtype != torch.int32 else b)
