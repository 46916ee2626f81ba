"""Paged cache: values of very unequal size.  Rows of zeros (exponent 0 in the 8-bit format) among small values must not cost the others
their bits.  Tolerance and definition: tests/cache_util.py."""
import pytest
import torch

from tests.cache_util import Cache, attention, check, decoded, forward, routed

pytestmark = pytest.mark.gpu


def zeros_among(L, size, every):
    x = torch.full((L, 1, 1), size, dtype=torch.float64)
    x[::every] = 0.0
    return x


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads", [(28, 4, 128), (8, 1, 64)])
@pytest.mark.parametrize("size", [1e-6, 1e-10, 1e-30])
@pytest.mark.parametrize("new", [1, 5])
def test_zero_rows_among_small_values(kind, heads, size, new):
    """Every fifth value row is zeros, inside the window and before it; then all of them."""
    Hq, Hkv, D = heads
    L = 500
    for every in (5, 1):
        c = Cache(kind, 32, Hkv, D, [L, L], 23, v_scale=zeros_among(L, size, every))
        d = routed(2 * new, 0.6, new)
        O, Q = forward(c, Hq, [new] * 2, 100, d=d, seed=2)
        want, bound = attention(c, Q, [new] * 2, d, 100)
        check(O, want, bound, f"{kind} {heads} values {size}, zeros every {every}")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,lengths,new", [((28, 4, 128), [500, 300], [40, 40]), ((28, 4, 128), [700, 700], [300, 230]),
                                               ((8, 1, 64), [500], [60])])
@pytest.mark.parametrize("size", [1e-6, 1e-10, 1e-30])
def test_zero_rows_among_small_values_chunks(kind, heads, lengths, new, size):
    Hq, Hkv, D = heads
    for every in (5, 1):
        c = Cache(kind, 32, Hkv, D, [max(lengths)] * len(lengths), 23, v_scale=zeros_among(max(lengths), size, every))
        d = routed(sum(new), 0.6, new[0])
        O, Q = forward(c, Hq, new, 100, d=d, seed=2)
        want, bound = attention(c, Q, new, d, 100)
        check(O, want, bound, f"{kind} {heads} values {size}, zeros every {every}")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("new", [5, 40, 300])
@pytest.mark.parametrize("size", [2.0 ** 22, 1e15, 1e30])
def test_values_of_later_tokens(kind, new, size):
    """The values of the last two tokens are `size` times the others': nothing of that reaches the rows before them."""
    L, Hq, Hkv, D, W = 600, 28, 4, 128, 60
    x = torch.full((L, 1, 1), 1e-5, dtype=torch.float64)
    x[-2:] *= size
    c = Cache(kind, 64, Hkv, D, [L, L], 24, v_scale=x)
    d = routed(2 * new, 0.6, new)
    O, Q = forward(c, Hq, [new] * 2, W, d=d, seed=2)
    want, bound = attention(c, Q, [new] * 2, d, W)
    check(O, want, bound, f"{kind} new {new} size {size}")


@pytest.mark.parametrize("new", [40, 300])
def test_sizes_from_one_end_of_the_range_to_the_other(new):
    """Values of 1e-36 and of 1e36 side by side, keys of 1e-20 to 1e3: the sums of the weights know nothing of them."""
    L, Hq, Hkv, D, W = 600, 28, 4, 128, 150
    g = torch.Generator().manual_seed(9)
    v = 10.0 ** (torch.randint(0, 5, (L, 1, 1), generator=g).double() * 18 - 36)
    v[:200] = 1e36
    v[200:520] = 1e-36
    k = 10.0 ** torch.randint(-20, 1, (L, 1, 1), generator=g).double()
    c = Cache("e4m3", 16, Hkv, D, [L, L], 25, v_scale=v, k_scale=k)
    d = routed(2 * new, 0.6, new)
    O, Q = forward(c, Hq, [new] * 2, W, d=d, seed=2)
    want, bound = attention(c, Q, [new] * 2, d, W)
    check(O, want, bound, f"new {new}")


@pytest.mark.parametrize("heads,lengths,new", [((28, 4, 128), [700, 300], [30, 40]), ((28, 4, 128), [700, 300], [230, 40]), ((8, 1, 64), [900], [100]),
                                               ((16, 16, 64), [1800, 1500], [1400, 100])])
def test_chunks_from_8_bits_equal_those_from_what_they_stand_for(heads, lengths, new):
    """The same bits as from a bf16 cache of the decoded values: whole chunks, elements of Q of every size, an infinite one."""
    Hq, Hkv, D = heads
    c = Cache("e4m3", 64, Hkv, D, lengths, 26)
    b = Cache("bf16", 64, Hkv, D, lengths, 26)
    for i, n in enumerate(lengths):
        j = torch.arange(n, device="cuda")
        pages = b.table[i].long()[j // 64]
        b.poolK[pages, :, j % 64] = c.K[i].bfloat16()
        b.poolV[pages, :, j % 64] = c.V[i].bfloat16()
    N = sum(new)
    g = torch.Generator().manual_seed(4)
    Q = torch.randn((N, Hq, D), generator=g) * 2.0 ** torch.randint(-30, 3, (N, Hq, D), generator=g)
    Q[3, 1, 7] = float("inf")
    Q = Q.bfloat16().cuda()
    d = routed(N, 0.6, 1)
    a = forward(c, Hq, new, 100, d=d, Q=Q)[0]
    w = forward(b, Hq, new, 100, d=d, Q=Q)[0]
    assert torch.equal(a.view(torch.int16), w.view(torch.int16)) or (
        torch.equal(a.isnan(), w.isnan()) and torch.equal(a.nan_to_num(), w.nan_to_num()))
    assert bool(a[3, 1].isnan().any()) and not bool(a[0].isnan().any())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 70, 400])
def test_every_code_with_every_exponent(D, new):
    """A window of the token itself: its result is its value row as it stands, rounded to bf16 (in the path of few rows, of chunks and
    of chunks from a decoded copy).  All 254 codes that are numbers, all exponents that a row can have."""
    Hkv, page = 4, 64
    L = 512
    c = Cache("e4m3", page, Hkv, D, [L], 27)
    g = torch.Generator().manual_seed(new + D)
    codes = torch.arange(L * Hkv * D, dtype=torch.int64).view(L, Hkv, D) % 254
    codes = (codes + (codes >= 127).long()).to(torch.uint8)                       # all but 127 and 255
    exps = (torch.arange(L * Hkv).view(L, Hkv) % 246 + 1).to(torch.uint8)         # 1 .. 246 (448 * 2^120 is no bf16)
    exps = exps[torch.randperm(L, generator=g)]
    if new == 1:
        exps = exps.clamp(20, 230)                         # (a lone weight's accumulator is fp32 times 2^e on its way)
    j = torch.arange(L)
    pages = c.table[0].cpu().long()[j // page]
    for h in range(Hkv):
        c.poolV[pages.cuda(), h, (j % page).cuda()] = codes[:, h].cuda()
        c.vs[pages.cuda(), h, (j % page).cuda()] = exps[:, h].cuda()
    G = 4 if new == 400 else 1
    Q = torch.randn((new, G * Hkv, D), generator=g).bfloat16().cuda()
    O = forward(c, G * Hkv, [new], 0, Q=Q)[0]
    want = torch.from_numpy(decoded(codes.numpy(), exps.numpy()))[L - new:].cuda()
    assert torch.equal(O, want.bfloat16().repeat_interleave(G, 1))
