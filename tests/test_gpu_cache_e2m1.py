"""4-bit paged caches: the write of new tokens (every bit) and the read back against the format's definition, and the attention over
them against its definition in 64 bits (tests/cache_util.py has the tolerance)."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_e2m1_util import Cache4, decoded4, quantise4
from tests.cache_util import attention, check, forward, routed

pytestmark = pytest.mark.gpu

HEADS = [(28, 4, 128), (32, 8, 128), (12, 2, 64), (4, 4, 64), (8, 1, 128)]


def special_rows(D):
    """Rows at the edges of the format: zeros, turning points of the exponent, ties of scales and codes, blocks that round to nothing,
    the ends of bf16, values that are not finite."""
    r = np.random.default_rng(5)
    x = r.standard_normal((20, D))
    x[0] = 0.0
    x[1] = -0.0
    x[2] = np.clip(x[2], -2.6, 2.6); x[2, 0] = 2.625                  # 2688 * 2^-10: the largest of its exponent
    x[3] = np.clip(x[3], -2.6, 2.6); x[3, 0] = 2.640625               # the next bf16
    x[4] *= 2.0 ** np.arange(D).clip(max=40)[::-1]                   # blocks of very unequal sizes
    x[5] = 2.0 ** -130 * np.sign(x[5])                               # below the least exponent
    x[6] *= 1e-38
    x[7] = np.clip(x[7], -1, 1) * 3e38
    x[8, 5] = np.inf; x[8, 6] = -np.inf
    x[9, 1] = np.nan
    x[10] = np.inf
    x[11] = np.nan
    x[12] = (np.arange(D) % 27 - 13) / 2; x[12, 0] = 2688            # a large block beside ties of codes at scales that are rounded
    x[13] = 2.0 ** -133
    x[14] = 2688 * 2.0 ** -126
    x[15, 0] = 3.3895313892515355e38                                 # the largest bf16
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for i, s in enumerate((1.0, 1.125, 1.875, 11 / 8)):              # every tie, for scales of one to four bits
        x[16 + i] = np.resize(np.concatenate([ties, -ties]), D) * s
    x[19, 16:32] = 2.0 ** -16                                        # a block whose scale rounds to zero beside one of 1344
    x[19, 0] = 1344.0
    return torch.from_numpy(x).bfloat16()


def append_and_compare(page, Hkv, D, lengths, new, interleaved, uniform=False):
    c = Cache4(page, Hkv, D, lengths, seed=page + D, interleaved=interleaved)
    N = sum(new)
    g = torch.Generator().manual_seed(N)
    rows = {x: (torch.randn((N, Hkv, D), generator=g) * torch.exp(2 * torch.randn((N, Hkv, D // 16), generator=g)).repeat_interleave(16, -1)).bfloat16()
            for x in "KV"}
    s = special_rows(D)[:N]
    rows["K"][:len(s), 0] = s
    rows["V"][N - len(s):, Hkv - 1] = s
    fused = torch.zeros((N, 3 * Hkv, D), dtype=torch.bfloat16)       # strided inputs: slices of one projection's output
    fused[:, Hkv:2 * Hkv], fused[:, 2 * Hkv:] = rows["K"], rows["V"]
    fused = fused.cuda()
    want = [x.cpu().clone() for x in (c.poolK, c.poolV, c.ks, c.vs)]
    p = l2a.params(len(new), max(new), max(lengths), 2 * Hkv, Hkv, D, 100, k_stride=(0, 3 * Hkv * D), v_stride=(0, 3 * Hkv * D))
    cu = None if uniform else torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    l2a.l2a_cache_append(p, c.handle, fused[:, Hkv:], fused[:, 2 * Hkv:], cu, N)
    torch.cuda.synchronize()
    table = c.table.cpu().long()
    t = 0
    for b, n in enumerate(new):
        pos = torch.arange(lengths[b] - n, lengths[b])
        at, slot = table[b, pos // page], pos % page
        for i, x in enumerate("KV"):
            q, s, e = quantise4(rows[x][t:t + n].double().numpy())
            want[i][at, :, slot] = torch.from_numpy(q)
            want[2 + i][at, :, slot] = torch.from_numpy(e)
            want[2 + i][:, :, page:].unflatten(2, (page, D // 16))[at, :, slot] = torch.from_numpy(s)
        t += n
    for a, b in zip(want, (c.poolK, c.poolV, c.ks, c.vs)):           # new slots and all others
        assert torch.equal(a, b.cpu())


@pytest.mark.parametrize("page,Hkv,D,lengths,new", [
    (16, 1, 128, [1], [1]),
    (16, 2, 64, [16, 17, 33], [16, 1, 20]),
    (32, 4, 128, [100, 5, 64, 31], [37, 0, 64, 1]),
    (64, 8, 128, [1000, 64, 65], [333, 1, 2]),
    (128, 3, 64, [128, 129, 500], [128, 129, 9]),
    (64, 2, 128, [3 + i for i in range(70)], [i % 3 for i in range(70)]),
    (64, 1, 128, [6000, 900], [5001, 0]),                            # more tokens than a wave of small CTAs
])
def test_append_writes_the_formats_bits(page, Hkv, D, lengths, new):
    append_and_compare(page, Hkv, D, lengths, new, interleaved=page == 64)


def test_append_of_as_many_tokens_each():
    append_and_compare(32, 2, 64, [40, 33, 20], [20, 20, 20], False, uniform=True)


@pytest.mark.parametrize("page,Hkv,D,lengths,misaligned", [(16, 2, 64, [1, 16, 40], False), (64, 3, 128, [500, 64, 3], True), (128, 1, 128, [700], False)])
def test_read_gives_what_the_cache_stands_for(page, Hkv, D, lengths, misaligned):
    c = Cache4(page, Hkv, D, lengths, seed=D, interleaved=page == 64)
    B, Lk, off = len(lengths), max(lengths) + 5, 8 if misaligned else 0
    c = Cache4(page, Hkv, D, lengths, seed=D, interleaved=page == 64, per=-(-Lk // page))
    first = torch.tensor([(-3, 0, 2)[b % 3] for b in range(B)], dtype=torch.int32).cuda()
    out = [torch.full((B * Lk * Hkv * D + off,), float("nan"), device="cuda", dtype=torch.bfloat16)[off:].view(B, Lk, Hkv, D) for _ in "KV"]
    l2a.l2a_cache_read(l2a.params(B, 1, Lk, Hkv, Hkv, D, 0), c.handle, first, *out)
    for got, true in zip(out, (c.K, c.V)):
        for b in range(B):
            want = torch.zeros((Lk, Hkv, D), dtype=torch.float64, device="cuda")
            f = int(first[b])
            n = lengths[b] - max(f, 0)
            want[max(-f, 0):max(-f, 0) + n] = true[b][max(f, 0):]
            assert torch.equal(got[b].double(), want)


def test_values_that_are_not_finite_come_back_as_nan_of_their_block():
    c = Cache4(16, 1, 64, [2], seed=1)
    x = torch.randn((2, 1, 64)).bfloat16()
    x[0, 0, 5], x[1, 0, 40] = float("inf"), float("nan")
    p = l2a.params(1, 2, 2, 1, 1, 64, 0)
    l2a.l2a_cache_append(p, c.handle, x.cuda(), x.cuda(), None, 2)
    out = torch.empty((1, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    l2a.l2a_cache_read(p, c.handle, None, out, torch.empty_like(out))
    want = decoded4(*quantise4(x.double().numpy()))
    assert np.array_equal(out[0].double().cpu().numpy(), want, equal_nan=True)
    assert out[0, 0, 0, :16].isnan().all() and not out[0, 0, 0, 16:].isnan().any() and out[0, 1, 0, 32:48].isnan().all()


# ---------------------------------------------------------------------------------------------------------- attention
def run(page, Hq, Hkv, D, W, lengths, new, density, seed, **kw):
    c = Cache4(page, Hkv, D, lengths, seed, **kw)
    d = routed(sum(new), density, seed)
    O, Q = forward(c, Hq, new, W, d=d, seed=seed)
    want, size = attention(c, Q, new, d, W)
    check(O, want, size, f"page {page} {Hq}/{Hkv}x{D} W {W} {lengths} new {new}")


@pytest.mark.parametrize("page,heads,W,lengths,density", [
    (16, HEADS[0], 4096, [1], 1.0),
    (16, HEADS[1], 0, [1, 2, 17, 64, 65], 0.5),
    (64, HEADS[0], 100, [63, 64, 65, 127, 128, 129], 1.0),
    (32, HEADS[2], 128, [500, 3, 129, 130, 257], 0.5),
    (128, HEADS[4], 1000, [5000, 100, 1001, 1002, 2003], 0.6),
    (64, HEADS[3], 64, [9001, 1], 1.0),
    (16, HEADS[1], 4096, [12000, 4097, 4098, 300], 0.5),
    (64, HEADS[0], 4096, [70000, 20], 1.0),
    (128, (2, 2, 128), 31, [64, 1000], 0.0),
    (32, (16, 1, 64), 200, [700, 33], 0.5),
    (32, (24, 1, 128), 200, [700, 33], 0.5),
])
def test_one_token_per_sequence(page, heads, W, lengths, density):
    run(page, *heads, W, lengths, [1] * len(lengths), density, seed=sum(lengths) + page)


@pytest.mark.parametrize("page,heads,W,lengths,new,density", [
    (16, HEADS[3], 10, [20, 30], [16, 17], 0.5),
    (64, HEADS[0], 100, [300, 40, 7], [2, 3, 7], 0.4),
    (32, HEADS[1], 64, [200, 128, 129], [5, 32, 33], 0.3),
    (128, HEADS[4], 128, [600, 32, 300], [16, 32, 33], 0.3),
    (16, HEADS[2], 128, [2000], [200], 0.2),
    (64, HEADS[0], 128, [700, 700], [700, 0], 0.2),
    (64, HEADS[1], 4096, [900, 5000], [300, 64], 0.2),
    (16, HEADS[0], 1000, [3000, 1, 2500, 64, 1100], [129, 1, 1, 64, 500], 0.25),
    (128, HEADS[2], 0, [300], [130], 0.5),
    (32, HEADS[3], 100000, [513], [257], 0.5),
    (64, HEADS[1], 200, [1200], [600], 1.0),
    (64, HEADS[1], 200, [1200], [600], 0.0),
    (32, HEADS[0], 4096, [33000, 9000], [5, 5], 0.3),
    (64, HEADS[0], 200, [2000, 70], [220, 70], 0.3),
    (64, (40, 1, 128), 64, [600, 20], [1, 20], 0.5),
    (16, (80, 1, 64), 64, [300, 20], [1, 7], 0.5),
    (128, (32, 8, 64), 300, [1500, 400], [300, 300], 0.3),
])
def test_chunks(page, heads, W, lengths, new, density):
    run(page, *heads, W, lengths, new, density, seed=sum(lengths) + page)


@pytest.mark.parametrize("new", [[1, 1], [3, 1], [60, 20]])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_and_blocks_of_very_unequal_sizes(D, new):
    """Keys and values between 2^-20 and 2^20 times the others, rows and blocks of zeros among them."""
    def rows(which, b, x):
        n = x.shape[0]
        f = torch.exp2(((torch.arange(n) * 7) % 41 - 20).float())[:, None, None] if which else torch.ones((n, 1, 1))
        x = x * f
        x[3::11] = 0
        x[5::13, :, 16:32] = 0
        x[6::13, :, :16] *= 2.0 ** -12
        return x.bfloat16()
    c = Cache4(32, 2, D, [300, 90], 3, rows=rows, spread=0.0)
    d = routed(sum(new), 0.6, 3)
    O, Q = forward(c, 8, new, 40, d=d, seed=3)
    want, size = attention(c, Q, new, d, 40)
    check(O, want, size, f"unequal {new}")


def test_the_workspace_without_the_copy_gives_the_same_bits():
    Hq, Hkv, D, W, lengths, new = 28, 4, 128, 200, [2000, 900], [220, 100]
    c = Cache4(64, Hkv, D, lengths, 9)
    d = routed(sum(new), 0.3, 9)
    O, Q = forward(c, Hq, new, W, d=d, seed=9)
    p = l2a.params(2, max(new), max(lengths), Hq, Hkv, D, W)
    bf16 = l2a.L2ACache.from_buffer_copy(c.handle)
    bf16.kind, bf16.page_stride = l2a.CACHE_BF16, 0
    least, most = (l2a.l2a_cache_workspace_bytes(p, h, sum(new)) for h in (bf16, c.handle))
    assert least < most
    ws = torch.empty(least, dtype=torch.uint8, device="cuda")
    O2 = torch.empty_like(O)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    l2a.l2a_cache_forward(p, c.handle, Q, cu, sum(new), d, O2, ws)
    assert torch.equal(O, O2)


@pytest.mark.parametrize("new", [[1, 1], [60, 20]])
def test_modules_one_at_a_time(new):
    Hq, Hkv, D, W, lengths, N = 28, 4, 128, 64, [400, 90], sum(new)
    c, c2 = Cache4(32, Hkv, D, lengths, 1), Cache4(64, Hkv, D, lengths, 2)
    d = routed(N, 0.4, 3)
    S, Q = forward(c, Hq, new, W, d=d, flags=l2a.FLAG_SKIP_GLOBAL)
    want, size = attention(c, Q, new, 0 * d, W)
    check(S, want, size, "s")
    A, _ = forward(c2, Hq, new, W, d=d, Q=Q, flags=l2a.FLAG_SKIP_LOCAL)
    a, size_a = attention(c2, Q, new, d, W, local=False)
    check(A, a, size_a, "d a")
    O, _ = forward(c2, Hq, new, W, d=d, Q=Q, O=S, flags=l2a.FLAG_GLOBAL_PHASE)
    check(O, a + S.double(), size_a, "s + d a")
    assert torch.equal(O[d == 0], S[d == 0])


@pytest.mark.parametrize("new", [[1, 1], [300, 20]])
def test_captured_call_follows_the_lengths(new):
    Hq, Hkv, D, W = 32, 8, 128, 100
    c = Cache4(64, Hkv, D, [900, 500], 4)
    N = sum(new)
    Q, d = torch.randn((N, Hq, D), device="cuda").bfloat16(), routed(N, 0.5, 4)
    p = l2a.params(2, max(new), 900, Hq, Hkv, D, W)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, c.handle, N), dtype=torch.uint8, device="cuda")
    O = torch.zeros_like(Q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        l2a.l2a_cache_forward(p, c.handle, Q, cu, N, d, O, ws)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        l2a.l2a_cache_forward(p, c.handle, Q, cu, N, d, O, ws)
    for lengths in ([900, 500], [700, 321], [300, 500]):
        c.length.copy_(torch.tensor(lengths, dtype=torch.int32))
        g.replay()
        c.lengths, K, V = lengths, c.K, c.V
        c.K, c.V = [k[:n] for k, n in zip(K, lengths)], [v[:n] for v, n in zip(V, lengths)]
        want, size = attention(c, Q, new, d, W)
        check(O, want, size, f"{lengths}")
        c.K, c.V = K, V
