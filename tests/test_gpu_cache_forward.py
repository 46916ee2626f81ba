"""Attention over the paged cache against its definition in 64 bits (tests/cache_util.py has the tolerance)."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import Cache, attention, check, forward, routed

pytestmark = pytest.mark.gpu

HEADS = [(28, 4, 128), (32, 8, 128), (12, 2, 64), (4, 4, 64), (8, 1, 128)]


def run(kind, page, Hq, Hkv, D, W, lengths, new, density, seed, **kw):
    c = Cache(kind, page, Hkv, D, lengths, seed, **kw)
    d = routed(sum(new), density, seed)
    O, Q = forward(c, Hq, new, W, d=d, seed=seed)
    want, size = attention(c, Q, new, d, W)
    check(O, want, size, f"{kind} page {page} {Hq}/{Hkv}x{D} W {W} {lengths} new {new}")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("page,heads,W,lengths,density", [
    (16, HEADS[0], 4096, [1], 1.0),
    (16, HEADS[1], 0, [1, 2, 17, 64, 65], 0.5),                # no neighbour: s = v
    (64, HEADS[0], 100, [63, 64, 65, 127, 128, 129], 1.0),
    (32, HEADS[2], 128, [500, 3, 129, 130, 257], 0.5),
    (128, HEADS[4], 1000, [5000, 100, 1001, 1002, 2003], 0.6),
    (64, HEADS[3], 64, [9001, 1], 1.0),
    (16, HEADS[1], 4096, [12000, 4097, 4098, 300], 0.5),
    (64, HEADS[0], 4096, [9001], 1.0),
    (64, HEADS[0], 4096, [70000, 20], 1.0),
    (128, (2, 2, 128), 31, [64, 1000], 0.0),
    (32, (16, 1, 64), 200, [700, 33], 0.5),                    # sixteen heads of a group
    (32, (24, 1, 128), 200, [700, 33], 0.5),                   # more than sixteen
])
def test_one_token_per_sequence(kind, page, heads, W, lengths, density):
    run(kind, page, *heads, W, lengths, [1] * len(lengths), density, seed=sum(lengths) + page)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("page,heads,W,lengths,new,density", [
    (16, HEADS[3], 10, [20, 30], [16, 17], 0.5),               # 16 and 17 rows of a head group
    (64, HEADS[0], 100, [300, 40, 7], [2, 3, 7], 0.4),
    (32, HEADS[1], 64, [200, 128, 129], [5, 32, 33], 0.3),     # 128 and 132 rows
    (128, HEADS[4], 128, [600, 32, 300], [16, 32, 33], 0.3),
    (16, HEADS[2], 128, [2000], [200], 0.2),
    (64, HEADS[0], 128, [700, 700], [700, 0], 0.2),            # a whole prompt, and a sequence without new tokens
    (64, HEADS[1], 4096, [900, 5000], [300, 64], 0.2),
    (16, HEADS[0], 1000, [3000, 1, 2500, 64, 1100], [129, 1, 1, 64, 500], 0.25),       # chunks and single tokens in one call
    (128, HEADS[2], 0, [300], [130], 0.5),
    (32, HEADS[3], 100000, [513], [257], 0.5),                 # the window sees everything
    (64, HEADS[1], 200, [1200], [600], 1.0),
    (64, HEADS[1], 200, [1200], [600], 0.0),
    (16, HEADS[4], 4096, [20000], [50], 0.2),
    (32, HEADS[0], 4096, [33000, 9000], [5, 5], 0.3),
    (64, HEADS[1], 300, [9000] * 8, [12] * 8, 0.3),            # four blocks of rows cost more than the path of the chunks
    (16, HEADS[0], 200, [3000, 2500], [146, 147], 0.5),        # 1022 and 1029 rows
    (128, HEADS[1], 200, [3000, 70], [256, 70], 0.3),
    (64, HEADS[0], 200, [2000, 70], [219, 70], 0.3),           # 1533 rows
    (64, HEADS[0], 200, [2000, 70], [220, 70], 0.3),           # 1540
    (64, (2, 1, 128), 500, [40 + 7 * i for i in range(40)], [1 + 3 * (i % 5) for i in range(40)], 0.3),
    (16, (4, 1, 64), 64, [3 + i for i in range(1100)], [1 + i % 3 for i in range(1100)], 0.5),      # more sequences than the plans keep on chip
    (64, (40, 1, 128), 64, [600, 20], [1, 20], 0.5),           # 40 heads of a group
    (64, (80, 1, 64), 64, [300, 20], [1, 7], 0.5),
])
def test_chunks(kind, page, heads, W, lengths, new, density):
    run(kind, page, *heads, W, lengths, new, density, seed=sum(lengths) + page)


def _random(n, seed):
    r = np.random.default_rng(seed)
    out = []
    for i in range(n):
        heads = HEADS[r.integers(len(HEADS))]
        B = int(r.integers(1, 6))
        lengths = [int(2 ** r.uniform(0, 12.5)) for _ in range(B)]
        new = [min(x, int(2 ** r.uniform(0, 9))) if r.random() < 0.6 else min(1, x) for x in lengths]
        if r.random() < 0.3:
            new[r.integers(B)] = 0
        if sum(new) == 0:
            new[0] = 1
        out.append(("e4m3" if r.random() < 0.6 else "bf16", int(r.choice([16, 32, 64, 128])), heads,
                    int(r.choice([0, 1, 63, 128, 1000, 4096])), lengths, new, float(r.choice([0.0, 0.1, 0.5, 1.0])), i))
    return out


@pytest.mark.parametrize("kind,page,heads,W,lengths,new,density,seed", _random(24, 20260317))
def test_random(kind, page, heads, W, lengths, new, density, seed):
    run(kind, page, *heads, W, lengths, new, density, seed=seed)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("lengths,new", [([400, 90, 1000], [1, 1, 1]), ([400, 90, 1000], [150, 20, 1])])
def test_modules_one_at_a_time(kind, lengths, new):
    """SKIP_GLOBAL gives s, SKIP_LOCAL d a, and GLOBAL_PHASE on another cache adds d a to what O holds, rows not routed untouched."""
    Hq, Hkv, D, W, N = 28, 4, 128, 64, sum(new)
    c, c2 = Cache(kind, 32, Hkv, D, lengths, 1), Cache(kind, 64, Hkv, D, lengths, 2)
    d = routed(N, 0.4, 3)
    S, Q = forward(c, Hq, new, W, d=d, flags=l2a.FLAG_SKIP_GLOBAL)
    want, size = attention(c, Q, new, 0 * d, W)
    check(S, want, size, "s")
    S0, _ = forward(c, Hq, new, W, d=None, Q=Q)
    assert torch.equal(S, S0)
    A, _ = forward(c2, Hq, new, W, d=d, Q=Q, flags=l2a.FLAG_SKIP_LOCAL)
    a, size_a = attention(c2, Q, new, d, W, local=False)
    check(A, a, size_a, "d a")
    assert not A[d == 0].any()
    O, _ = forward(c2, Hq, new, W, d=d, Q=Q, O=S, flags=l2a.FLAG_GLOBAL_PHASE)
    check(O, a + S.double(), size_a, "s + d a")
    assert torch.equal(O[d == 0], S[d == 0])


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("lengths,new", [([700, 300], [1, 1]), ([700, 300], [60, 20])])
def test_pages_before_the_window_may_be_gone(kind, lengths, new):
    """No token routed: what lies wholly before every window is not read, nor its table entry."""
    Hq, Hkv, D, W = 32, 8, 128, 100
    c = Cache(kind, 16, Hkv, D, lengths, 5)
    want = forward(c, Hq, new, W, d=None)[0].clone()
    for b in range(2):
        gone = max(0, lengths[b] - new[b] - W) // 16
        pages = c.table[b, :gone].long()
        for pool in (c.poolK, c.poolV):
            pool[pages] = float("nan") if kind == "bf16" else 0x7f
        c.table[b, :gone] = torch.tensor([-1, 1 << 30], dtype=torch.int32).cuda().repeat(gone)[:gone]
    assert torch.equal(forward(c, Hq, new, W, d=None)[0], want)


@pytest.mark.parametrize("new", [1, 40])
def test_uniform_new_tokens_need_no_list(new):
    c = Cache("e4m3", 64, 4, 128, [500, 80, 41], 6)
    d = routed(3 * new, 0.5, 1)
    a, Q = forward(c, 28, [new] * 3, 100, d=d)
    b, _ = forward(c, 28, [new] * 3, 100, d=d, Q=Q, uniform=True)
    assert torch.equal(a, b)


@pytest.mark.parametrize("lengths,new", [([0, 5], [0, 1]), ([2, 5], [4, 1]), ([0, 3], [2, 2]), ([30, 40], [60, 20])])
def test_rows_without_a_key_are_zeros(lengths, new):
    """More new tokens than the sequence is long: those at positions below 0 see nothing."""
    c = Cache("bf16", 16, 4, 64, [max(1, x) for x in lengths], 8, per=8)
    c.length.copy_(torch.tensor(lengths))
    d = torch.ones(sum(new), dtype=torch.uint8, device="cuda")
    O, Q = forward(c, 4, new, 8, d=d, Lk=128)
    t = 0
    for b, n in enumerate(new):
        bad = max(0, n - lengths[b])
        assert not O[t:t + bad].any()
        assert O[t + bad:t + n].any(-1).all()
        t += n


@pytest.mark.parametrize("new", [1, 33])
def test_strided_tensors(new):
    """Q as a slice of a fused projection, O as columns of a wider buffer, K and V in one allocation."""
    Hq, Hkv, D, W = 28, 4, 128, 64
    lengths = [300, 90]
    c = Cache("e4m3", 16, Hkv, D, lengths, 4, interleaved=True)
    d = routed(2 * new, 0.5, 4)
    want, Q = forward(c, Hq, [new] * 2, W, d=d)
    N = 2 * new
    fused = torch.randn((N, Hq + 2 * Hkv, D), device="cuda", dtype=torch.bfloat16)
    fused[:, :Hq] = Q
    wide = torch.full((N, Hq + 1, D), 7.0, device="cuda", dtype=torch.bfloat16)
    p = l2a.params(2, new, 300, Hq, Hkv, D, W, q_stride=(0, (Hq + 2 * Hkv) * D), o_stride=(0, (Hq + 1) * D))
    ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, c.handle, N), dtype=torch.uint8, device="cuda")
    l2a.l2a_cache_forward(p, c.handle, fused, None, N, d, wide, ws)
    assert torch.equal(wide[:, :Hq], want) and bool((wide[:, Hq] == 7).all())


@pytest.mark.parametrize("new", [1, 30])
def test_captured_calls_follow_the_lengths(new):
    """A captured append + attention replays with the lengths, pages and tokens of the moment; on a stream of its own."""
    Hq, Hkv, D, W, B = 28, 4, 128, 64, 2
    c = Cache("e4m3", 16, Hkv, D, [400, 300], 11)
    p = l2a.params(B, new, 400, Hq, Hkv, D, W)
    N = B * new
    ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, c.handle, N), dtype=torch.uint8, device="cuda")
    Q, K, V = (torch.zeros((N, h, D), device="cuda", dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    d = torch.zeros(N, dtype=torch.uint8, device="cuda")
    O = torch.empty_like(Q)

    def step():
        l2a.l2a_cache_append(p, c.handle, K, V, None, N)
        l2a.l2a_cache_forward(p, c.handle, Q, None, N, d, O, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ([400, 300], [new, 200], [100, new], [399, 64 + new]):
        c.length.copy_(torch.tensor(lengths))
        for x in (Q, K, V):
            x.normal_()
        d.copy_(routed(N, 0.5, lengths[0]))
        graph.replay()
        got = O.clone()
        dense = [torch.empty((B, 400, Hkv, D), device="cuda", dtype=torch.bfloat16) for _ in "KV"]
        l2a.l2a_cache_read(p, c.handle, None, *dense)
        c.lengths = lengths
        c.K, c.V = ([x[b, :lengths[b]].double() for b in range(B)] for x in dense)
        want, size = attention(c, Q, [new] * B, d, W)
        check(got, want, size, f"replay at {lengths}")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("new", [1, 40])
def test_large_and_small_scales(kind, new):
    """Keys and values far from one, scores of hundreds: exponents of every kind, sharp and flat soft-max."""
    for k, v, scale in ((1e-4, 1e-6, 0.0), (30.0, 1e5, 0.0), (1.0, 1e30, 0.5), (1e-20, 1e-30, 1e19), (1e6, 1.0, 1e-6)):
        c = Cache(kind, 32, 4, 128, [300, 700], 12, k_scale=k, v_scale=v)
        d = routed(2 * new, 0.5, 1)
        O, Q = forward(c, 28, [new] * 2, 100, d=d, scale=scale)
        want, size = attention(c, Q, [new] * 2, d, 100, scale=scale or None)
        # a score of size s carries D 2^-24 s in fp32, more than the docstring's 2^-12 where the scores are hundreds
        top = max(float((Q.double().abs().amax() * x.abs().amax() * (scale or 128 ** -0.5) * 128 ** 0.5)) for x in c.K)
        check(O, want, size * (1 + 2.0 ** 8 * 2 * 128 ** 0.5 * 2.0 ** -23 * top), f"scales {k} {v} {scale}")


def test_same_bits_again():
    c = Cache("e4m3", 64, 4, 128, [9000, 1000, 40], 13)
    for new in ([1, 1, 1], [300, 40, 1]):
        d = routed(sum(new), 0.3, 2)
        a, Q = forward(c, 28, new, 500, d=d)
        for _ in range(3):
            assert torch.equal(forward(c, 28, new, 500, d=d, Q=Q)[0], a)
