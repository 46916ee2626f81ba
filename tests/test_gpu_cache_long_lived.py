"""Appending, attending, weighing and evicting in turns, as a server does: every result against the definitions on what the cache holds
at that time; and the example server with 4-bit caches, whole and bounded."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import decoded4, make_cache, quantise4
from tests.cache_util import attention, check, decoded, quantise, routed
from tests.cache_weigh_util import weights as weights_of
from tests.test_gpu_cache_evict import stays

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def rounded(kind, x):
    """What a cache of the kind stands for, of rows in 64 bits."""
    if kind == "bf16":
        return x
    coded = quantise4(x.cpu().numpy()) if kind == "e2m1" else quantise(x.cpu().numpy())
    return torch.from_numpy((decoded4 if kind == "e2m1" else decoded)(*coded)).to(x.device)


@pytest.mark.parametrize("kind", ["e2m1", "e4m3", "bf16"])
def test_a_cache_that_is_shortened_as_it_grows(kind):
    Hq, Hkv, D, W, page, B = 8, 2, 128, 50, 16, 2
    most, keep, first = 400, 150, 4
    c = make_cache(kind, page, Hkv, D, [0, 0], 1, per=-(-most // page))
    big = make_cache(kind, page, Hkv, D, [most] * (2 * B), 1)                 # pools for twice the sequences
    tables = [big.table[:B].contiguous(), big.table[B:].contiguous()]
    length = torch.zeros(B, dtype=torch.int32, device="cuda")

    def handle(table):
        K, V = (x.view(torch.float4_e2m1fn_x2) if kind == "e2m1" else x for x in (big.poolK, big.poolV))
        return l2a.cache(K, V, table, length, k_scale=big.ks, v_scale=big.vs)
    w = torch.full((big.poolK.shape[0], Hkv, page), float("nan"), device="cuda")
    K = [torch.zeros((0, Hkv, D), dtype=torch.float64, device="cuda") for _ in range(B)]
    V, weight = [x.clone() for x in K], [torch.zeros((0, Hkv), dtype=torch.float64, device="cuda") for _ in range(B)]
    slack = [x.clone() for x in weight]                                       # bound of the weights' error
    now, held = 0, [0, 0]
    for step, new in enumerate([[120, 40], [1, 1], [90, 30], [1, 1], [60, 100], [5, 3], [100, 120], [1, 1]]):
        N = sum(new)
        g = torch.Generator().manual_seed(step)
        q, k, v = ((torch.randn((N, h, D), generator=g)).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
        d = routed(N, 0.6, step)
        held = [n + x for n, x in zip(held, new)]
        length.copy_(torch.tensor(held, dtype=torch.int32))
        cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
        p, h = l2a.params(B, max(new), most, Hq, Hkv, D, W), handle(tables[now])
        O = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(l2a.l2a_cache_workspace_bytes(p, h, N), l2a.l2a_cache_weigh_workspace_bytes(p, h, N)), dtype=torch.uint8, device="cuda")
        l2a.l2a_cache_append(p, h, k, v, cu, N)
        l2a.l2a_cache_forward(p, h, q, cu, N, d, O, ws)
        l2a.l2a_cache_weigh(p, h, q, cu, N, d, w, ws)
        t = 0
        for b, n in enumerate(new):
            K[b] = torch.cat([K[b], rounded(kind, k[t:t + n].double())])
            V[b] = torch.cat([V[b], rounded(kind, v[t:t + n].double())])
            t += n
        c.K, c.V, c.lengths = K, V, held
        want, size = attention(c, q, new, d, W)
        check(O, want, size, f"step {step}")
        for b, (inc, off) in enumerate(weights_of(c, q, new, d)):
            zeros = torch.zeros((new[b], Hkv), dtype=torch.float64, device="cuda")
            weight[b] = torch.cat([weight[b], zeros]) + inc
            slack[b] = torch.cat([slack[b], zeros]) + off + 2.0 ** -24 * weight[b]
            j = torch.arange(held[b], device="cuda")
            got = w[tables[now][b, j // page].long(), :, j % page].double()
            assert bool(((got - weight[b]).abs() <= slack[b] + 1e-36).all())
        if max(held) <= 200:
            continue
        pe = l2a.params(B, keep, most, Hq, Hkv, D, W)
        kept = torch.empty((B, Hkv, keep), dtype=torch.int32, device="cuda")
        ws = torch.empty(l2a.l2a_cache_evict_workspace_bytes(pe, h), dtype=torch.uint8, device="cuda")
        old = [w[tables[now][b, torch.arange(held[b], device="cuda") // page].long(), :, torch.arange(held[b], device="cuda") % page].double() for b in range(B)]
        l2a.l2a_cache_evict(pe, h, w, torch.full((B,), keep, dtype=torch.int32, device="cuda"), first, W, handle(tables[1 - now]), w, length, kept, ws)
        now = 1 - now
        for b in range(B):
            m = min(held[b], keep)
            rows = torch.stack([torch.tensor(stays(old[b][:, x].cpu().numpy(), held[b], keep, first, W, keep), device="cuda") for x in range(Hkv)], 1)
            assert torch.equal(kept[b, :, :m].T.long(), rows) and int(length[b]) == m
            heads = torch.arange(Hkv, device="cuda")
            K[b], V[b] = K[b][rows, heads], V[b][rows, heads]
            weight[b], slack[b] = old[b][rows, heads], torch.zeros((m, Hkv), dtype=torch.float64, device="cuda")
            held[b] = m
    assert step == 7 and max(held) <= 200


def example():
    spec = importlib.util.spec_from_file_location("paged_serving", os.path.join(ROOT, "examples", "paged_serving.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_server_with_4_bits_equals_the_layer_over_whole_sequences():
    prompts, answer, heads, window = [1500, 130, 700, 1], 6, (28, 4, 128), 256
    layer, out, dec, data = example().serve(prompts, answer, heads=heads, window=window, chunk=600, bits=4, seed=3)
    Hq, Hkv, D = heads
    for s, n in enumerate(prompts):
        L = n + answer
        (Q, _, _), (Qg, _, _) = data[s]
        (K, V), (Kg, Vg) = layer.take_out(s)              # the layer on what the caches stand for
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
        assert bool(((got - want).abs() <= 2 * 2.0 ** -8 * 2 * vmax + 4 * 2.0 ** -8 * want.abs()).all())


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_the_server_with_a_bound(bits):
    prompts, answer, window, bound = [1500, 130, 700], 30, 128, 500
    layer, out, dec, _ = example().serve(prompts, answer, heads=(8, 2, 128), window=window, chunk=300, bits=bits, seed=3, bound=bound)
    n_pages = layer.local.K.shape[0]
    assert all(torch.isfinite(o.float()).all() for o in out) and [len(o) for o in out] == [n + answer for n in prompts]
    assert max(layer.held) <= bound and layer.lengths.tolist() == layer.held
    pages = sum(-(-n // layer.page) for n in layer.held)
    assert len(layer.free) == n_pages - pages and len(set(layer.free)) == len(layer.free)
    assert torch.isfinite(layer.weights[layer.table[0, :-(-layer.held[0] // layer.page)].long()]).all()
