"""The example server (chunks and single tokens mixed, caches in pages, router between the modules) against the layer over whole
sequences: l2a_forward_sets with the decisions that the server took."""
import importlib.util
import os

import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import Cache, check, forward

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("paged_serving", os.path.join(ROOT, "examples", "paged_serving.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [16, 8])
def test_server_equals_the_layer_over_whole_sequences(bits):
    prompts, answer, heads, window = [1500, 130, 700, 1], 6, (28, 4, 128), 256
    layer, out, dec, data = example().serve(prompts, answer, heads=heads, window=window, chunk=600, bits=bits, seed=3)
    assert 0 < sum(int(d.sum()) for d in dec) < sum(len(d) for d in dec)
    Hq, Hkv, D = heads
    for s, n in enumerate(prompts):
        L = n + answer
        (Q, K, V), (Qg, Kg, Vg) = data[s]
        if bits == 8:                                    # the layer on what the caches stand for
            (K, V), (Kg, Vg) = layer.take_out(s)
        else:
            for got, want in zip(layer.take_out(s), ((K, V), (Kg, Vg))):
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        p = l2a.params(1, L, L, Hq, Hkv, D, window)
        buf = l2a.Buffers.allocate(p)
        buf.router.copy_(dec[s][None])
        buf.route()
        l2a.l2a_forward_sets(p, *(x[None].contiguous() for x in (Q, K, V, Qg, Kg, Vg)), buf.d_mask, buf.q_idx, buf.n_routed, buf.prefix,
                             buf.O, None, None, None, None, buf.fwd_ws)
        torch.cuda.synchronize()
        want, got = buf.O[0].double(), out[s].double()
        # both sides round the weights (2^-8 of sum P |v| each, at most max |v|), s and the sum (2^-8 each)
        vmax = max(float(V.abs().max()), float(Vg.abs().max()))
        bound = 2 * 2.0 ** -8 * 2 * vmax + 4 * 2.0 ** -8 * want.abs()
        assert bool(((got - want).abs() <= bound).all())
        assert float((got - want).norm()) <= 2.0 ** -7 * float(want.norm())      # independent roundings of 2^-9 on average, several
    assert len(layer.free) == layer.local.K.shape[0]


def test_offsets_beyond_2_31():
    """A pool of over 2^31 elements: pages at its end are written, attended to and read."""
    Hkv, page, D, n_pages = 8, 128, 128, 20000               # 2.6e9 codes
    pool = [torch.zeros((n_pages, Hkv, page, D), dtype=torch.uint8, device="cuda") for _ in "KV"]
    exps = [torch.full((n_pages, Hkv, page), 127, dtype=torch.uint8, device="cuda") for _ in "KV"]
    small = Cache("e4m3", page, Hkv, D, [700, 300], 21)
    order = torch.tensor([n_pages - 1 - 2 * i for i in range(8)] + [3, 4], device="cuda")
    table = torch.stack([order[:6], order[4:10]]).int()
    table[1, :3] = order[6:9].int()
    for b, n in ((0, 6), (1, 3)):
        for i in range(n):
            for big, x in zip(pool + exps, (small.poolK, small.poolV, small.ks, small.vs)):
                big[table[b, i]] = x[small.table[b, i]]
    handle = l2a.cache(*pool, table.contiguous(), small.length, *exps)
    for new in ([1, 1], [5, 3], [300, 40]):
        d = torch.ones(sum(new), dtype=torch.uint8, device="cuda")
        want, Q = forward(small, 32, new, 100, d=d)
        far = Cache.__new__(Cache)
        far.__dict__.update(small.__dict__, handle=handle)
        got, _ = forward(far, 32, new, 100, d=d, Q=Q)
        assert torch.equal(got, want)
    p = l2a.params(2, 1, 700, 32, Hkv, D, 100)
    dense = [[torch.empty((2, 700, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in "KV"] for _ in range(2)]
    l2a.l2a_cache_read(p, small.handle, None, *dense[0])
    l2a.l2a_cache_read(p, handle, None, *dense[1])
    assert torch.equal(dense[0][0], dense[1][0]) and torch.equal(dense[0][1], dense[1][1])
    x = torch.randn((2, Hkv, D), device="cuda", dtype=torch.bfloat16)
    for h in (small.handle, handle):
        l2a.l2a_cache_append(p, h, x, x, None, 2)
    assert torch.equal(pool[0][table[0, 5]], small.poolK[small.table[0, 5]]) and torch.equal(exps[1][table[1, 2]], small.vs[small.table[1, 2]])
