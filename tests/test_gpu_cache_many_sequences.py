"""Paged cache: more sequences in a call than a grid has rows, and host bounds (Lk) under which the tiles of all sequences together pass
2^31: the path of the few rows takes such calls in several launches."""
import pytest
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import Cache, attention, check, routed
from tests.test_gpu_cache_bounds import tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("listed", [False, True])
def test_more_sequences_than_a_grid_has_rows(listed):
    """70001 sequences of up to 16 tokens, one page and (with a list, but for every seventh) one new token each."""
    B, D, W, page = 70001, 64, 3, 16
    g = torch.Generator(device="cuda").manual_seed(4)
    K, V = (torch.randn((B, 1, page, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "KV")
    table = torch.randperm(B, generator=g, device="cuda").int()[:, None].contiguous()
    length = torch.randint(1, page + 1, (B,), generator=g, device="cuda").int()
    new = (torch.arange(B, device="cuda") % 7 != 0).int() if listed else torch.ones(B, dtype=torch.int32, device="cuda")
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), new.cumsum(0).int()]) if listed else None
    N = int(new.sum())
    Q = torch.randn((N, 1, D), generator=g, device="cuda", dtype=torch.bfloat16)
    d = (torch.rand(N, generator=g, device="cuda") < 0.5).to(torch.uint8)
    c = l2a.cache(K, V, table, length)
    p = l2a.params(B, 1, page, 1, 1, D, W)
    ws = torch.full((l2a.l2a_cache_workspace_bytes(p, c, N),), 0xA5, dtype=torch.uint8, device="cuda")
    O = torch.full_like(Q, float("nan"))
    l2a.l2a_cache_forward(p, c, Q, cu, N, d, O, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    b = torch.arange(B, device="cuda")[new > 0]
    Kd, Vd = (x[table[b, 0].long(), 0].double() for x in (K, V))
    s = torch.einsum("nd,njd->nj", Q[:, 0].double(), Kd) / D ** 0.5
    j, pos = torch.arange(page, device="cuda")[None], (length[b] - 1)[:, None]
    want = torch.zeros((N, D), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for seen, weight in (((j <= pos) & (j >= pos - W), 1.0), (j <= pos, d.double()[:, None])):
        x = torch.softmax(s.masked_fill(~seen, -float("inf")), 1)
        want += weight * torch.einsum("nj,njd->nd", x, Vd)
        size += weight * torch.einsum("nj,njd->nd", x, Vd.abs())
    check(O[:, 0], want, size, f"{B} sequences, list: {listed}")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
@pytest.mark.parametrize("new", [[1] * 300, [1 + b % 3 for b in range(300)]])
def test_tiles_of_the_bounds_pass_32_bits(kind, new):
    """300 sequences of 8 heads, each of at most 2^26 tokens: 2.5e9 tiles of 64 keys if they were that long."""
    B, Hq, Hkv, D, W, Lk = 300, 16, 8, 64, 40, 1 << 26
    c = Cache(kind, 128, Hkv, D, [3 + b % 90 for b in range(B)], 6)
    table = torch.full((B, Lk // 128), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.handle = l2a.cache(c.poolK, c.poolV, table, c.length, k_scale=c.ks, v_scale=c.vs)
    N, uniform = sum(new), len(set(new)) == 1
    Q = torch.randn((N, Hq, D), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    d = routed(N, 0.5, 1)
    p = l2a.params(B, max(new), Lk, Hq, Hkv, D, W)
    ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, c.handle, N), dtype=torch.uint8, device="cuda")
    O = torch.full_like(Q, float("nan"))
    l2a.l2a_cache_forward(p, c.handle, Q, None if uniform else tokens(new), N, d, O, ws)
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    check(O, *attention(c, Q, new, d, W), f"{kind} bounds of 2^26 tokens")


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_units_of_work_of_the_bounds_pass_32_bits(kind):
    """32 sequences of 8 heads, each of at most 2^26 tokens, a chunk of each: the sums of the plan are 64 bits wide, the result that of
    the call with close bounds."""
    B, Hq, Hkv, D, W, Lk, new = 32, 32, 8, 64, 40, 1 << 26, 20
    c = Cache(kind, 128, Hkv, D, [new + b % 90 * 7 for b in range(B)], 7)
    N = B * new
    Q = torch.randn((N, Hq, D), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    d = routed(N, 0.5, 1)
    table = torch.full((B, Lk // 128), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    far = l2a.cache(c.poolK, c.poolV, table, c.length, k_scale=c.ks, v_scale=c.vs)
    out = []
    for handle, keys in ((c.handle, max(c.lengths)), (far, Lk)):
        p = l2a.params(B, new, keys, Hq, Hkv, D, W)
        ws = torch.empty(l2a.l2a_cache_workspace_bytes(p, handle, N), dtype=torch.uint8, device="cuda")
        O = torch.full_like(Q, float("nan"))
        l2a.l2a_cache_forward(p, handle, Q, None, N, d, O, ws)
        torch.cuda.synchronize()
        assert l2a.l2a_workspace_status(ws) == 0
        out.append(O)
    check(out[0], *attention(c, Q, [new] * B, d, W), kind)
    assert torch.equal(out[0], out[1])
