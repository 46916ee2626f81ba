"""Paged cache: the write of new tokens (bits of codes and exponents) and the read back, against the format's definition."""
import numpy as np
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import Cache, decoded, quantise

pytestmark = pytest.mark.gpu


def special_rows(D):
    """Rows at the edges of the format: zeros, the exponent's turning points, subnormal codes, the ends of bf16, not finite values."""
    r = np.random.default_rng(5)
    x = r.standard_normal((16, D))
    x[0] = 0.0
    x[1, 3] = -0.0
    x[2] = np.clip(x[2], -3.4, 3.4); x[2, 0] = 3.5                 # 448 * 2^-7: the largest of its exponent
    x[3] = np.clip(x[3], -3.4, 3.4); x[3, 0] = 3.515625            # the next bf16
    x[4] *= 2.0 ** np.arange(D).clip(max=40)[::-1]                # a wide row: most values round to zero
    x[5] = 2.0 ** -130 * np.sign(x[5])                            # below the least exponent
    x[6] *= 1e-38
    x[7] = np.clip(x[7], -1, 1) * 3e38
    x[8, 5] = np.inf; x[8, 6] = -np.inf
    x[9, 1] = np.nan
    x[10] = np.inf
    x[11] = np.nan
    x[12, :] = (np.arange(D) % 17 - 8) / 16 + 1 / 32; x[12, 0] = 448          # ties of subnormal codes at 2^e = 1
    x[13] = 2.0 ** -133
    x[14] = 448 * 2.0 ** -126
    x[15, 0] = 3.3895313892515355e38                              # the largest bf16
    return torch.from_numpy(x).bfloat16()


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("page,Hkv,D,lengths,new", [
    (16, 1, 128, [1], [1]),
    (16, 2, 64, [16, 17, 33], [16, 1, 20]),
    (32, 4, 128, [100, 5, 64, 31], [37, 0, 64, 1]),
    (64, 8, 128, [1000, 64, 65], [333, 1, 2]),
    (128, 3, 64, [128, 129, 500], [128, 129, 9]),
    (64, 2, 128, [3 + i for i in range(70)], [i % 3 for i in range(70)]),      # more sequences than lanes
])
def test_append_writes_the_formats_bits(kind, page, Hkv, D, lengths, new):
    c = Cache(kind, page, Hkv, D, lengths, seed=page + D, interleaved=page == 64 and Hkv == 8)
    N = sum(new)
    g = torch.Generator().manual_seed(N)
    rows = {x: torch.randn((N, Hkv, D), generator=g).bfloat16() for x in "KV"}
    s = special_rows(D)[:N]
    rows["K"][:len(s), 0] = s
    rows["V"][N - len(s):, Hkv - 1] = s
    # strided inputs: slices of one projection's output
    fused = torch.zeros((N, 3 * Hkv, D), dtype=torch.bfloat16)
    fused[:, Hkv:2 * Hkv], fused[:, 2 * Hkv:] = rows["K"], rows["V"]
    fused = fused.cuda()
    before = [x.cpu() if x is not None else None for x in (c.poolK, c.poolV, c.ks, c.vs)]
    p = l2a.params(len(new), max(new), max(lengths), 2 * Hkv, Hkv, D, 100, k_stride=(0, 3 * Hkv * D), v_stride=(0, 3 * Hkv * D))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    l2a.l2a_cache_append(p, c.handle, fused[:, Hkv:], fused[:, 2 * Hkv:], cu, N)
    torch.cuda.synchronize()
    table = c.table.cpu().long()
    t = 0
    for b, n in enumerate(new):
        pos = torch.arange(lengths[b] - n, lengths[b])
        at, slot = table[b, pos // page], pos % page
        for i, x in enumerate("KV"):
            if kind == "bf16":
                before[i][at, :, slot] = rows[x][t:t + n]
            else:
                code, e = quantise(rows[x][t:t + n].double().numpy())
                before[i][at, :, slot] = torch.from_numpy(code)
                before[2 + i][at, :, slot] = torch.from_numpy(e)
        t += n
    for want, got in zip(before, (c.poolK, c.poolV, c.ks, c.vs)):       # new slots and all others
        if want is not None:
            a, b = (x.contiguous().view(torch.int16) if kind == "bf16" and x.dtype == torch.bfloat16 else x for x in (want, got.cpu()))
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("Hkv,D,misaligned", [(1, 64, False), (3, 128, True)])
def test_append_and_read_of_many_tokens(kind, Hkv, D, misaligned):
    """More tokens than a wave of small CTAs; with tensors that start at 16 bytes, not 32."""
    lengths, new = [6000, 900], [5001, 0]
    c = Cache(kind, 64, Hkv, D, lengths, seed=D)
    N, off = sum(new), 8 if misaligned else 0
    rows = [torch.randn(N * Hkv * D + off, device="cuda").bfloat16()[off:].view(N, Hkv, D) for _ in "KV"]
    p = l2a.params(2, 5001, 6000, Hkv, Hkv, D, 0)
    cu = torch.tensor([0, 5001, 5001], dtype=torch.int32).cuda()
    l2a.l2a_cache_append(p, c.handle, *rows, cu, N)
    out = [torch.empty(2 * 6000 * Hkv * D + off, device="cuda", dtype=torch.bfloat16)[off:].view(2, 6000, Hkv, D) for _ in "KV"]
    l2a.l2a_cache_read(p, c.handle, None, *out)
    for x, got, old in zip(rows, out, (c.K, c.V)):
        want = x.double().cpu().numpy()
        if kind == "e4m3":
            want = decoded(*quantise(want))
        assert np.array_equal(got[0, 999:].double().cpu().numpy(), want)
        assert torch.equal(got[0, :999].double(), old[0][:999]) and torch.equal(got[1, :900].double(), old[1])
        assert not got[1, 900:].any()


def test_append_of_one_length_without_a_list():
    c = Cache("e4m3", 16, 2, 128, [40, 40, 40], seed=1)
    p = l2a.params(3, 4, 40, 2, 2, 128, 8)
    x = torch.randn((12, 2, 128), device="cuda", dtype=torch.bfloat16)
    l2a.l2a_cache_append(p, c.handle, x, x, None, 12)
    for b in range(3):
        for i in range(4):
            code, e = quantise(x[4 * b + i].double().cpu().numpy())
            page = int(c.table[b, (36 + i) // 16])
            assert np.array_equal(c.poolK[page, :, (36 + i) % 16].cpu().numpy(), code)
            assert np.array_equal(c.vs[page, :, (36 + i) % 16].cpu().numpy(), e)


def test_append_out_of_bounds_values_write_nothing():
    """Lengths past Lk, new tokens ahead of position 0, table entries that are no page: no slot changes outside the sequence's own."""
    c = Cache("e4m3", 16, 1, 64, [32, 32], seed=3)
    before = c.poolK.clone()
    c.length.copy_(torch.tensor([33, 2]))                          # past Lk; three new tokens of a sequence of two
    c.table[1, 0] = 1 << 20
    p = l2a.params(2, 3, 32, 1, 1, 64, 8)
    x = torch.ones((6, 1, 64), device="cuda", dtype=torch.bfloat16)
    l2a.l2a_cache_append(p, c.handle, x, x, None, 6)
    torch.cuda.synchronize()
    changed = (c.poolK != before).any(-1).any(1).cpu()             # [pages, slots]
    want = torch.zeros_like(changed)
    want[int(c.table[0, 1]), 14:16] = True                        # positions 30, 31; 32 is past Lk
    assert torch.equal(changed, want)


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("page,Hkv,D,lengths,first", [
    (16, 1, 128, [1], None),
    (16, 3, 64, [0, 17, 100], None),
    (64, 8, 128, [700, 64, 65], [600, 0, -3]),
    (128, 2, 128, [129, 1000], [1, 999]),
    (32, 4, 64, [33, 32, 31, 5000], None),
])
def test_read_gives_what_the_cache_stands_for(kind, page, Hkv, D, lengths, first):
    c = Cache(kind, page, Hkv, D, lengths, seed=page * D, interleaved=page == 128, k_scale=1e-3, v_scale=1e4)
    B, Lk = len(lengths), max(lengths)
    p = l2a.params(B, 1, Lk, Hkv, Hkv, D, 0, k_stride=(0, 2 * Hkv * D), v_stride=(Lk * Hkv * D + 64, 0))
    K = torch.full((B, Lk, 2, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    V = torch.full((B, Lk * Hkv * D + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    f = None if first is None else torch.tensor(first, dtype=torch.int32).cuda()
    l2a.l2a_cache_read(p, c.handle, f, K, V)
    torch.cuda.synchronize()
    assert K[:, :, 1].isnan().all() and V[:, Lk * Hkv * D:].isnan().all()
    got = {"K": K[:, :, 0], "V": V[:, :Lk * Hkv * D].view(B, Lk, Hkv, D)}
    for b in range(B):
        start = 0 if first is None else first[b]
        for x, true in (("K", c.K[b]), ("V", c.V[b])):
            want = torch.zeros((Lk, Hkv, D), dtype=torch.float64, device="cuda")
            for t in range(Lk):
                if 0 <= start + t < lengths[b]:
                    want[t] = true[start + t]
            assert torch.equal(got[x][b].double(), want), (b, x)


def test_what_is_appended_is_read():
    """Round trip through the calls alone, error of a value within the format's bound: half a step, 2^-4 relative, or 2^-10 * 2^e."""
    lengths = [77, 200]
    c = Cache("e4m3", 32, 4, 128, lengths, seed=9)
    p = l2a.params(2, 200, 200, 4, 4, 128, 0)
    cu = torch.tensor([0, 77, 277], dtype=torch.int32).cuda()
    x = (torch.randn((277, 4, 128), device="cuda") * 7).bfloat16()
    l2a.l2a_cache_append(p, c.handle, x, x, cu, 277)
    K = torch.empty((2, 200, 4, 128), dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    l2a.l2a_cache_read(p, c.handle, None, K, V)
    got = torch.cat([K[0, :77], K[1]]).double()
    top = x.double().abs().amax(-1, keepdim=True)
    bound = torch.maximum(2.0 ** -4 * x.double().abs(), 2.0 ** -10 * top / 224)          # 2^e < top / 224
    assert bool(((got - x.double()).abs() <= bound).all()) and torch.equal(K, V)
