"""Eviction from a paged cache against its definition: which positions stay, and every bit of what moves."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache

pytestmark = pytest.mark.gpu


def stays(w, n, keep, sinks, recent, most):
    """Positions of one head that stay, from the definition."""
    m = min(n, max(keep, 0), most)
    r = min(recent, m)
    f = min(sinks, m - r)
    middle = range(f, n - r)
    rank = sorted(middle, key=lambda j: (0, -w[j], j) if not np.isnan(w[j]) else (1, 0, j))
    return [*range(f), *sorted(rank[:m - f - r]), *range(n - r, n)]


def raw(x):
    """Bytes of a pool, the same number of dimensions."""
    return x if x.dtype == torch.uint8 else x.contiguous().view(torch.uint8)


class Target:
    """Pages for what stays, in pools of their own; slots hold a pattern."""

    def __init__(self, c, most, page, seed=7):
        g = torch.Generator().manual_seed(seed)
        B, per = len(c.lengths), max(1, -(-most // page))
        n_pages = B * per + 1
        self.page, self.most = page, most
        self.table = torch.randperm(n_pages, generator=g)[:B * per].view(B, per).int().cuda()
        shape = (n_pages, c.Hkv, page)

        def pool(x, last):
            if x is None:
                return None
            full = shape + (last,) if last else shape[:2] + (page * x.shape[2] // c.page,)
            return torch.full(full, 0x5A, dtype=torch.uint8).view(x.dtype).cuda()
        width = {"bf16": 2 * c.D, "e4m3": c.D, "e2m1": c.D // 2}[c.kind]
        self.K, self.V, self.ks, self.vs = pool(c.poolK, width), pool(c.poolV, width), pool(c.ks, 0), pool(c.vs, 0)
        self.w = torch.full(shape, -7.0, device="cuda")
        self.lengths = torch.full((B,), -5, dtype=torch.int32, device="cuda")
        kv = (x.view(torch.float4_e2m1fn_x2) if c.kind == "e2m1" else x for x in (self.K, self.V))
        self.handle = l2a.cache(*kv, self.table, self.lengths, k_scale=self.ks, v_scale=self.vs)


def rows_of(c, K, scales, table, page, b, g, pos):
    """(codes, exponents, block scales) of the tokens at `pos` of head g of sequence b."""
    pos = torch.as_tensor(pos, dtype=torch.long, device="cuda")
    at, slot = table[b, pos // page].long(), pos % page
    out = [raw(K)[at, g, slot]]
    if scales is not None:
        out.append(scales[at, g, slot])
        if c.kind == "e2m1":
            out.append(scales[:, :, page:].unflatten(2, (page, c.D // 16))[at, g, slot])
    return out


def run(kind, page, to_page, Hkv, D, lengths, keep, sinks, recent, most=None, weights=None, seed=1, interleaved=False, Lk=None, with_kept=True):
    most = max(1, max(keep)) if most is None else most
    Lk = max(1, max(lengths)) if Lk is None else Lk
    c = make_cache(kind, page, Hkv, D, lengths, seed, interleaved=interleaved, per=-(-Lk // page))
    t = Target(c, most, to_page)
    n_pages = c.poolK.shape[0]
    g = torch.Generator().manual_seed(seed + 5)
    w = torch.rand((n_pages, Hkv, page), generator=g) if weights is None else weights(torch.rand((n_pages, Hkv, page), generator=g))
    w = w.cuda()
    p = l2a.params(len(lengths), most, Lk, Hkv, Hkv, D, 8)
    kept = torch.full((len(lengths), Hkv, most), -9, dtype=torch.int32, device="cuda") if with_kept else None
    nbytes = l2a.l2a_cache_evict_workspace_bytes(p, c.handle)
    ws = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    before = [raw(x).clone() for x in (c.poolK, c.poolV, w)]
    l2a.l2a_cache_evict(p, c.handle, w, torch.tensor(keep, dtype=torch.int32).cuda(), sinks, recent, t.handle, t.w, t.lengths, kept, ws[:nbytes])
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xA5).all())
    assert all(torch.equal(x, raw(y)) for x, y in zip(before, (c.poolK, c.poolV, w)))
    written = torch.zeros((t.K.shape[0], Hkv, to_page), dtype=torch.bool, device="cuda")
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            pos = torch.arange(n, device="cuda")
            wb = w[c.table[b, pos // page].long(), h, pos % page]
            want = stays(wb.double().cpu().numpy(), n, keep[b], sinks, recent, most)
            m = len(want)
            assert int(t.lengths[b]) == m
            if kept is not None:
                assert kept[b, h, :m].tolist() == want, (b, h)
                assert bool((kept[b, h, m:] == -1).all())
            for src, dst, es, ed in ((c.poolK, t.K, c.ks, t.ks), (c.poolV, t.V, c.vs, t.vs)):
                for x, y in zip(rows_of(c, src, es, c.table, page, b, h, want), rows_of(c, dst, ed, t.table, to_page, b, h, range(m))):
                    assert torch.equal(x, y)
            i = torch.arange(m, device="cuda")
            at = (t.table[b, i // to_page].long(), h, i % to_page)
            assert torch.equal(t.w[at].view(torch.int32), wb[torch.tensor(want, dtype=torch.long, device="cuda")].view(torch.int32))
            written[at] = True
    assert bool((t.w[~written] == -7.0).all()) and bool((raw(t.K)[~written] == 0x5A).all()) and bool((raw(t.V)[~written] == 0x5A).all())
    if t.ks is not None:
        assert bool((t.ks[:, :, :to_page][~written] == 0x5A).all())


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("page,to_page,Hkv,D,lengths,keep,sinks,recent", [
    (16, 16, 1, 128, [1], [1], 0, 0),
    (16, 32, 2, 64, [40, 17, 5], [20, 17, 9], 2, 8),
    (64, 64, 4, 128, [300, 64, 1], [150, 10, 1], 4, 32),
    (128, 16, 3, 64, [1000, 129, 0], [333, 128, 5], 0, 0),
    (32, 128, 8, 128, [500, 400], [499, 1], 4, 100),               # one token goes; the last tokens alone
    (64, 64, 2, 128, [9001, 4000], [4500, 0], 4, 1000),            # several CTAs of a cluster; nothing stays
    (16, 64, 1, 64, [33000], [1500], 1, 64),
])
def test_what_stays_and_moves(kind, page, to_page, Hkv, D, lengths, keep, sinks, recent):
    run(kind, page, to_page, Hkv, D, lengths, keep, sinks, recent, interleaved=page == 64)


@pytest.mark.parametrize("keep,sinks,recent,most", [([-3, 7, 100], 4, 4, 50), ([6, 8, 10], 4, 4, 10), ([30, 30, 30], 100, 0, 30),
                                                    ([30, 30, 30], 0, 100, 30), ([30, 30, 30], 10, 25, 30)])
def test_fewer_stay_than_are_always_kept(keep, sinks, recent, most):
    run("e4m3", 16, 16, 2, 64, [60, 60, 90], keep, sinks, recent, most=most)


def equal(w):
    return torch.zeros_like(w)


def few_values(w):
    return (w * 5).floor()


def zeros_of_both_signs(w):
    return torch.where(w < 0.3, -0.0, torch.where(w < 0.6, 0.0, w))


def special(w):
    x = (w - 0.5) * 1e-3
    for lo, v in ((0.0, float("nan")), (0.2, float("inf")), (0.3, float("-inf")), (0.4, 1e-42), (0.5, -1e-42), (0.6, 3e38), (0.65, -float("nan"))):
        x = torch.where((w >= lo) & (w < lo + 0.05), torch.tensor(v), x)
    return x


def close(w):
    """Neighbours in the last bits."""
    return (torch.tensor(1.0).view(torch.int32) + (w * 300).int()).view(torch.float32)


@pytest.mark.parametrize("weights", [equal, few_values, zeros_of_both_signs, special, close])
@pytest.mark.parametrize("length", [100, 20000])
def test_order_of_the_weights(weights, length):
    for keep in (length // 7, length // 2, length - 1):
        run("e2m1", 32, 32, 2, 64, [length], [keep], 3, 10, weights=weights)


def test_more_positions_than_shared_memory_keeps():
    run("e4m3", 128, 128, 1, 64, [450000], [200001], 4, 4096, weights=few_values)


def test_many_positions_in_shared_memory():
    run("e2m1", 128, 64, 1, 64, [300000, 1000], [120000, 900], 4, 4096)


def test_offsets_beyond_2_31():
    """Pools of over 2^31 bytes of codes: pages at their ends."""
    Hkv, page, D, n_pages = 8, 128, 128, 40000                        # 65536 bytes of codes a page
    small = make_cache("e2m1", page, Hkv, D, [700, 300], 21)
    codes = [torch.zeros((n_pages, Hkv, page, D // 2), dtype=torch.uint8, device="cuda") for _ in "KV"]
    scales = [torch.zeros((n_pages, Hkv, page * 9), dtype=torch.uint8, device="cuda") for _ in "KV"]
    weights = torch.zeros((n_pages, Hkv, page), device="cuda")
    w = torch.rand(small.poolK.shape[:3], device="cuda")
    src = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2, n_pages - 9, 5, n_pages - 5], [n_pages - 6, 4, n_pages - 7, 0, 0, 0]], device="cuda")
    for b, n in ((0, 6), (1, 3)):
        for i in range(n):
            for big, x in zip(codes + scales + [weights], (small.poolK, small.poolV, small.ks, small.vs, w)):
                big[src[b, i]] = x[small.table[b, i].long()]
    dst = torch.tensor([[n_pages - 20, n_pages - 21, n_pages - 22], [n_pages - 23, n_pages - 24, 7]], device="cuda")
    four = [x.view(torch.float4_e2m1fn_x2) for x in codes]
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    a, b = (l2a.cache(*four, t.int().contiguous(), n, *scales) for t, n in ((src, small.length), (dst, length)))
    target = Target(small, 384, page)
    p = l2a.params(2, 384, 700, Hkv, Hkv, D, 8)
    keep = torch.tensor([384, 200], dtype=torch.int32, device="cuda")
    ws = torch.empty(l2a.l2a_cache_evict_workspace_bytes(p, a), dtype=torch.uint8, device="cuda")
    kept = [torch.empty((2, Hkv, 384), dtype=torch.int32, device="cuda") for _ in range(2)]
    l2a.l2a_cache_evict(p, small.handle, w, keep, 4, 50, target.handle, target.w, target.lengths, kept[0], ws)
    l2a.l2a_cache_evict(p, a, weights, keep, 4, 50, b, weights, length, kept[1], ws)
    assert torch.equal(*kept) and length.tolist() == [384, 200]
    out = [[torch.empty((2, 384, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in "KV"] for _ in range(2)]
    pr = l2a.params(2, 1, 384, Hkv, Hkv, D, 0)
    l2a.l2a_cache_read(pr, target.handle, None, *out[0])
    l2a.l2a_cache_read(pr, b, None, *out[1])
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and bool(out[0][0].any())
    # attention and weights from the same places
    Q = torch.randn((2, 32, D), device="cuda").bfloat16()
    for new in (1, 40):
        pa = l2a.params(2, new, 384, 32, Hkv, D, 60)
        Q = torch.randn((2 * new, 32, D), device="cuda").bfloat16()
        d = torch.ones(2 * new, dtype=torch.uint8, device="cuda")
        got = []
        for h, x in ((target.handle, target.w), (b, weights)):
            O = torch.empty_like(Q)
            ws = torch.empty(max(l2a.l2a_cache_workspace_bytes(pa, h, 2 * new), l2a.l2a_cache_weigh_workspace_bytes(pa, h, 2 * new)), dtype=torch.uint8,
                             device="cuda")
            l2a.l2a_cache_forward(pa, h, Q, None, 2 * new, d, O, ws)
            l2a.l2a_cache_weigh(pa, h, Q, None, 2 * new, d, x, ws)
            table = target.table if h is target.handle else dst
            got.append((O, [x[table[s, torch.arange(n, device="cuda") // page].long(), :, torch.arange(n, device="cuda") % page]
                            for s, n in ((0, 384), (1, 200))]))
        assert torch.equal(got[0][0], got[1][0]) and all(torch.equal(x, y) for x, y in zip(got[0][1], got[1][1]))


def test_bounds_above_the_lengths():
    run("bf16", 64, 64, 2, 128, [100, 300], [50, 70], 2, 9, most=100, Lk=60000, with_kept=False)


def test_many_sequences():
    run("e2m1", 16, 16, 1, 64, [1 + i % 50 for i in range(300)], [1 + i % 23 for i in range(300)], 1, 3)


def test_a_captured_call_of_several_CTAs():
    c = make_cache("e4m3", 64, 1, 64, [40000], 3)
    t = Target(c, 9000, 64)
    w = torch.rand((c.poolK.shape[0], 1, 64), device="cuda")
    p = l2a.params(1, 9000, 40000, 1, 1, 64, 8)
    ws = torch.empty(l2a.l2a_cache_evict_workspace_bytes(p, c.handle), dtype=torch.uint8, device="cuda")
    kept = torch.zeros((1, 1, 9000), dtype=torch.int32, device="cuda")
    keep = torch.tensor([9000], dtype=torch.int32, device="cuda")
    l2a.l2a_cache_evict(p, c.handle, w, keep, 4, 100, t.handle, t.w, t.lengths, kept, ws)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        l2a.l2a_cache_evict(p, c.handle, w, keep, 4, 100, t.handle, t.w, t.lengths, kept, ws)
    for n in (40000, 20000, 8000):
        c.length.fill_(n)
        w.copy_(torch.rand_like(w))
        g.replay()
        torch.cuda.synchronize()
        j = torch.arange(n, device="cuda")
        want = stays(w[c.table[0, j // 64].long(), 0, j % 64].double().cpu().numpy(), n, 9000, 4, 100, 9000)
        assert kept[0, 0, :len(want)].tolist() == want and int(t.lengths) == len(want) and bool((kept[0, 0, len(want):] == -1).all())


def test_the_same_pools_and_lengths_in_place():
    """The other pages of the same pools, the lengths overwritten; captured and replayed on another stream."""
    page, Hkv, D, lengths, keep = 16, 2, 128, [200, 150], [90, 120]
    c = make_cache("e2m1", page, Hkv, D, [400, 400], 3)              # room in the pools
    table = c.table[:1, :].clone()
    src = torch.stack([table[0, :13], table[0, 12:25]]).contiguous()
    dst = c.table[1:, :16].reshape(2, 8).contiguous()
    length = torch.tensor(lengths, dtype=torch.int32).cuda()
    a, b = c.handle_of(src, length), c.handle_of(dst, length)
    w = torch.rand((c.poolK.shape[0], Hkv, page), device="cuda")
    pool = [x.clone() for x in (c.poolK, c.poolV, c.ks, c.vs, w)]
    p = l2a.params(2, 120, 208, Hkv, Hkv, D, 8)
    ws = torch.empty(l2a.l2a_cache_evict_workspace_bytes(p, a), dtype=torch.uint8, device="cuda")
    kept = torch.empty((2, Hkv, 120), dtype=torch.int32, device="cuda")
    k = torch.tensor(keep, dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        l2a.l2a_cache_evict(p, a, w, k, 2, 16, b, w, length, kept, ws)
    for _ in range(2):
        for x, y in zip((c.poolK, c.poolV, c.ks, c.vs, w), pool):
            x.copy_(y)
        length.copy_(torch.tensor(lengths, dtype=torch.int32))
        kept.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        assert length.tolist() == keep
        for s in range(2):
            for h in range(Hkv):
                pos = torch.arange(lengths[s], device="cuda")
                wb = pool[4][src[s, pos // page].long(), h, pos % page]
                want = stays(wb.double().cpu().numpy(), lengths[s], keep[s], 2, 16, 120)
                assert kept[s, h, :keep[s]].tolist() == want
                for x, y, e, f in ((pool[0], c.poolK, pool[2], c.ks), (pool[1], c.poolV, pool[3], c.vs)):
                    for u, v in zip(rows_of(c, x, e, src, page, s, h, want), rows_of(c, y, f, dst, page, s, h, range(keep[s]))):
                        assert torch.equal(u, v)
