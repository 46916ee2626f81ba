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


def test_bounds_above_the_lengths():
    run("bf16", 64, 64, 2, 128, [100, 300], [50, 70], 2, 9, most=100, Lk=60000, with_kept=False)


def test_many_sequences():
    run("e2m1", 16, 16, 1, 64, [1 + i % 50 for i in range(300)], [1 + i % 23 for i in range(300)], 1, 3)


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
