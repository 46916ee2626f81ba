"""Weights of the cached keys against their definition in 64 bits (tests/cache_weigh_util.py has the tolerance)."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import make_cache
from tests.cache_util import routed
from tests.cache_weigh_util import weigh, weights

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "e4m3", "e2m1"]
HEADS = [(28, 4, 128), (32, 8, 128), (12, 2, 64), (4, 4, 64), (8, 1, 128)]


def run(kind, page, heads, lengths, new, density, **kw):
    Hq, Hkv, D = heads
    seed = sum(lengths) + page
    c = make_cache(kind, page, Hkv, D, lengths, seed, interleaved=page == 64)
    d = None if density is None else routed(sum(new) + kw.get("extra", 0), density, seed)
    return weigh(c, Hq, new, d, seed=seed, **kw)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page,heads,lengths,density", [
    (16, HEADS[0], [1], 1.0),
    (16, HEADS[1], [1, 2, 17, 64, 65], 0.5),
    (64, HEADS[0], [63, 64, 65, 127, 128, 129], None),
    (32, HEADS[2], [500, 3, 129, 130, 257], 0.5),
    (128, HEADS[4], [5000, 100, 1001], 0.6),
    (64, HEADS[3], [9001, 1], 1.0),
    (16, HEADS[1], [12000, 4097, 300], 0.5),
    (64, HEADS[0], [40000, 20], 1.0),
    (64, HEADS[0], [300, 20], 0.0),                      # none counts: the new slots are zeros
    (32, (16, 1, 64), [700, 33], 0.5),
    (32, (24, 1, 128), [700, 33], None),                 # two blocks of rows
    (64, (80, 1, 64), [300, 20], 0.7),                   # more rows than one sequence keeps
])
def test_one_token_per_sequence(kind, page, heads, lengths, density):
    run(kind, page, heads, lengths, [1] * len(lengths), density)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page,heads,lengths,new,density", [
    (16, HEADS[3], [20, 30], [16, 17], 0.5),
    (64, HEADS[0], [300, 40, 7], [2, 3, 7], 0.4),
    (32, HEADS[1], [200, 128, 129], [5, 16, 17], 0.5),   # up to 64 rows, and 68
    (128, HEADS[4], [600, 32, 300], [16, 32, 33], 0.3),
    (16, HEADS[2], [2000], [200], 0.2),
    (64, HEADS[0], [700, 700], [700, 0], None),          # a whole prompt, and a sequence without new tokens
    (64, HEADS[1], [900, 5000], [300, 64], 0.2),
    (16, HEADS[0], [3000, 1, 2500, 64, 1100], [129, 1, 1, 64, 500], 0.25),
    (32, HEADS[3], [513], [257], 0.5),
    (64, HEADS[1], [1200], [600], 0.0),
    (32, HEADS[0], [20000, 9000], [5, 40], 0.3),
    (64, (2, 1, 128), [40 + 7 * i for i in range(40)], [1 + 3 * (i % 25) for i in range(40)], 0.3),
    (16, (4, 1, 64), [3 + i for i in range(1100)], [1 + i % 3 for i in range(1100)], 0.5),
    (64, (40, 1, 128), [600, 20], [1, 20], 0.5),
])
def test_chunks(kind, page, heads, lengths, new, density):
    run(kind, page, heads, lengths, new, density)


@pytest.mark.parametrize("kind", ["bf16", "e2m1"])
@pytest.mark.parametrize("lengths,new", [([300, 200], [7, 7]), ([900, 700], [300, 300])])
def test_as_many_tokens_each_scale_and_bounds(kind, lengths, new):
    run(kind, 32, HEADS[0], lengths, new, 0.5, uniform=True, scale=0.3)
    run(kind, 32, HEADS[0], lengths, new, 0.5, Lk=928 if lengths[0] == 900 else 320, Lq=400)


@pytest.mark.parametrize("new", [[3, 1], [100, 30]])
def test_rows_behind_the_last_sequence_and_several_calls(new):
    run("e4m3", 64, HEADS[1], [400, 90], new, 0.6, extra=9)
    run("e4m3", 64, HEADS[1], [400, 90], new, None, calls=3)


@pytest.mark.parametrize("new", [[2, 3], [150, 30]])
def test_strided_queries(new):
    c = make_cache("bf16", 32, 4, 128, [500, 90], 5)
    fused = torch.randn((sum(new), 36, 128), device="cuda").bfloat16()
    weigh(c, 28, new, routed(sum(new), 0.5, 1), Q=fused[:, :28])


@pytest.mark.parametrize("new", [[4], [200]])
def test_large_scores(new):
    """Scores of hundreds: one key takes nearly all, far ones underflow."""
    c = make_cache("bf16", 64, 2, 64, [700], 8, k_scale=30.0)
    weigh(c, 8, new, None, seed=3)


@pytest.mark.parametrize("new", [[1, 2], [90, 30]])
def test_a_row_of_nan_does_not_reach_other_sequences(new):
    c = make_cache("e2m1", 16, 2, 128, [300, 100], 8)
    Q = torch.randn((sum(new), 8, 128), device="cuda").bfloat16()
    Q[0, 3] = float("nan")                                            # the first head group of sequence 0
    w = torch.zeros((c.poolK.shape[0], 2, 16), device="cuda")
    p = l2a.params(2, max(new), 300, 8, 2, 128, 0)
    ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, sum(new)), dtype=torch.uint8, device="cuda")
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32).cuda()
    l2a.l2a_cache_weigh(p, c.handle, Q, cu, sum(new), None, w, ws)
    j = torch.arange(300, device="cuda")
    first = w[c.table[0, j // 16].long(), :, j % 16]
    assert first[:300 - new[0] + 1, 0].isnan().all() and torch.isfinite(first[:, 1]).all()
    j = j[:100]
    assert torch.isfinite(w[c.table[1, j // 16].long(), :, j % 16]).all()


@pytest.mark.parametrize("kind", ["bf16", "e2m1"])
@pytest.mark.parametrize("new", [[1, 1], [3, 50], [300, 20]])
def test_captured_calls_follow_their_inputs_and_give_the_same_bits(kind, new):
    Hq, Hkv, D = 32, 8, 128
    c = make_cache(kind, 64, Hkv, D, [900, 500], 4)
    N = sum(new)
    Q, d = torch.randn((N, Hq, D), device="cuda").bfloat16(), routed(N, 0.6, 4)
    d[0] = 1
    p = l2a.params(2, max(new), 900, Hq, Hkv, D, 0)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, N), dtype=torch.uint8, device="cuda")
    w = torch.zeros((c.poolK.shape[0], Hkv, 64), device="cuda")
    l2a.l2a_cache_weigh(p, c.handle, Q, cu, N, d, w, ws)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        l2a.l2a_cache_weigh(p, c.handle, Q, cu, N, d, w, ws)
    K = c.K
    for lengths in ([900, 500], [700, 321], [300, 500]):
        c.length.copy_(torch.tensor(lengths, dtype=torch.int32))
        c.lengths, c.K = lengths, [k[:n] for k, n in zip(K, lengths)]
        results = []
        for _ in range(2):
            w.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            results.append(w.clone())
        assert torch.equal(*results)
        for b, (inc, off) in enumerate(weights(c, Q, new, d)):
            j = torch.arange(lengths[b], device="cuda")
            got = w[c.table[b, j // 64].long(), :, j % 64].double()
            assert bool(((got - inc).abs() <= off + 2.0 ** -23 * inc).all())


def test_weights_of_a_softmax_sum_to_the_rows():
    """Every counted row gives one in all: long contexts, where few rows are divided among many CTAs, and blocks of rows among some."""
    for new in (1, 40):
        c = make_cache("e4m3", 128, 1, 64, [150000], 3)
        Q = torch.randn((new, 4, 64), device="cuda").bfloat16()
        p = l2a.params(1, new, 150000, 4, 1, 64, 0)
        ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(p, c.handle, new), dtype=torch.uint8, device="cuda")
        w = torch.zeros((c.poolK.shape[0], 1, 128), device="cuda")
        l2a.l2a_cache_weigh(p, c.handle, Q, None, new, None, w, ws)
        assert abs(float(w.double().sum()) / (4 * new) - 1) < 1e-5
