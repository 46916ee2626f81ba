"""Helpers for the tests of the paged cache: the 8-bit format and the attention over the cache, written plainly in 64 bits
and apart from the package, and a cache of random sequences on the GPU.

Tolerance of the attention, element by element.  bf16 has eight significant bits, so that rounding to it is off by at most half a
step, 2^-8 of the value.  With P the soft-max weights of a module, S = sum_j P_j |v_j| over what it sees:
  * the weights may enter the second product rounded to bf16 (the sum of the weights is taken before that): 2^-8 S;
  * fp32 scores: D products of bf16 or 8-bit numbers summed in fp32, |error| <= D 2^-24 sum |q_i k_i| scale, which for N(0, 1)
    inputs and D = 128 is below 128 2^-24 9 = 7e-5, and the same again for the exponentials and the sums: 2^-12 S together;
  * one rounding of the result to bf16, of a value that may be off by the above: 2^-8 (|o| + error).
So |err| <= 2^-8 |o| + (2^-8 + 2^-11) (S_local + d S_global)."""
import math

import numpy as np
import torch

from paper_2603_17484_b200 import l2a

CODE_VALUES = np.array([(-1.0 if c & 0x80 else 1.0) * ((c & 7) / 8 * 2.0 ** -6 if not (c >> 3) & 15 else
                                                       (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7))
                        for c in range(256)])
CODE_VALUES[0x7f] = CODE_VALUES[0xff] = np.nan


def quantise(rows):
    """(codes, exponents + 127) of rows [..., D] given in 64 bits, from the format's definition: nearest of the 127 magnitudes, a tie
    to the even code."""
    mag, sign = np.abs(rows), np.signbit(rows)
    finite = np.where(np.isfinite(mag), mag, 0.0)
    top = finite.max(-1)
    e = np.zeros(top.shape)
    some = top > 0
    f, x = np.frexp(top[some] / 448.0)              # top / 448 = f 2^x, f in [1/2, 1): exact, 448 = 7 * 2^6 needs the check below
    e[some] = np.where(np.ldexp(448.0, x - 1) >= top[some], x - 1, x)
    e = np.maximum(e, -126)
    y = mag / np.exp2(e)[..., None]
    table = CODE_VALUES[:127]
    hi = np.clip(np.searchsorted(table, np.where(np.isnan(y), 0.0, y)), 1, 126)
    lo = hi - 1
    with np.errstate(invalid="ignore"):
        d_lo, d_hi = y - table[lo], table[hi] - y
        code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(y), 127, code)
    return (code + np.where(sign & ~np.isnan(y), 128, 0)).astype(np.uint8), (e + 127).astype(np.uint8)


def decoded(codes, exponents):
    return CODE_VALUES[codes] * np.exp2(exponents.astype(np.float64) - 127)[..., None]


class Cache:
    """Sequences of given lengths in a shuffled pool.  Slots without a token hold NaN, table entries without a page a number that
    is none.  K, V: what the cache stands for, a list of [length, Hkv, D] in 64 bits on the GPU."""

    def __init__(self, kind, page, Hkv, D, lengths, seed, per=None, interleaved=False, k_scale=1.0, v_scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.page, self.Hkv, self.D, self.lengths = kind, page, Hkv, D, list(lengths)
        B = len(lengths)
        need = [-(-n // page) for n in lengths]
        per = max(1, max(need)) if per is None else per
        n_pages = sum(need) + 2
        order = torch.randperm(n_pages, generator=g)
        table = torch.randint(-(1 << 31), -1, (B, per), generator=g, dtype=torch.int64)
        table[:, ::2] = (1 << 31) - 1 - torch.arange(per)[::2]
        dtype = torch.bfloat16 if kind == "bf16" else torch.uint8
        shape = (n_pages, Hkv, page, D)
        pools = [torch.full((n_pages, 2, Hkv, page, D), float("nan") if kind == "bf16" else 0x7f, dtype=dtype)] * 2 if interleaved \
            else [torch.full(shape, float("nan") if kind == "bf16" else 0x7f, dtype=dtype) for _ in range(2)]
        if interleaved:
            pools = [pools[0][:, 0], pools[0][:, 1]]
        scales = [torch.full((n_pages, Hkv, page), 255, dtype=torch.uint8) for _ in range(2)]
        true = [[], []]
        at = 0
        for b, n in enumerate(lengths):
            pages = order[at:at + need[b]]
            at += need[b]
            table[b, :need[b]] = pages
            j = torch.arange(n)
            for which, factor in ((0, k_scale), (1, v_scale)):
                x = (torch.randn((n, Hkv, D), generator=g) * factor * torch.exp(0.5 * torch.randn((n, Hkv, 1), generator=g))).bfloat16()
                if kind == "bf16":
                    pools[which][pages[j // page], :, j % page] = x
                    true[which].append(x.double())
                else:
                    code, e = quantise(x.double().numpy())
                    pools[which][pages[j // page], :, j % page] = torch.from_numpy(code)
                    scales[which][pages[j // page], :, j % page] = torch.from_numpy(e)
                    true[which].append(torch.from_numpy(decoded(code, e)))
        if interleaved:
            both = torch.stack(pools, 1).cuda()
            self.poolK, self.poolV = both[:, 0], both[:, 1]
        else:
            self.poolK, self.poolV = pools[0].cuda(), pools[1].cuda()
        self.ks, self.vs = (None, None) if kind == "bf16" else (scales[0].cuda(), scales[1].cuda())
        self.table, self.length = table.int().cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
        self.K, self.V = [x.cuda() for x in true[0]], [x.cuda() for x in true[1]]
        self.handle = l2a.cache(self.poolK, self.poolV, self.table, self.length, k_scale=self.ks, v_scale=self.vs)


def attention(cache, Q, new, d, W, scale=None, local=True, only_global=False):
    """(o, bound) in 64 bits: o_t = s_t [local] + d_t a_t for the new tokens (new: how many of each sequence) on one token axis, and
    sum |P||v| of both modules, weighted the same."""
    N, Hq, D = Q.shape
    G = Hq // cache.Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    o = torch.zeros((N, Hq, D), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(o)
    t = 0
    for b, n in enumerate(new):
        length = cache.lengths[b]
        if n == 0:
            continue
        pos = torch.arange(length - n, length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")[None, :]
        dd = d[t:t + n].double()[:, None]
        for h in range(Hq):
            K, V = cache.K[b][:, h // G], cache.V[b][:, h // G]
            s = Q[t:t + n, h].double() @ K.T * scale
            for module, seen, weight in (("s", (j <= pos) & (j >= pos - W), torch.full_like(dd, float(local))),
                                         ("a", j <= pos, dd)):
                x = s.masked_fill(~seen, -math.inf)
                p = torch.exp(x - x.amax(1, keepdim=True).clamp(min=-1e300))
                p = p * seen / (p * seen).sum(1, keepdim=True).clamp(min=1e-300)
                o[t:t + n, h] += weight * (p @ V)
                size[t:t + n, h] += weight * (p @ V.abs())
        t += n
    return o, size


def check(got, want, size, what):
    """The bound of this module's docstring."""
    assert torch.isfinite(got.float()).all(), f"{what}: not finite"
    err = (got.double() - want).abs()
    bound = (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -11) * size).clamp(min=1e-300)
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1, f"{what}: {worst:.3f} times the bound at {np.unravel_index(int((err / bound).argmax()), err.shape)}"


def forward(cache, Hq, new, W, d=None, Q=None, seed=0, flags=0, Lk=None, Lq=None, O=None, uniform=False, scale=0.0):
    """One call on a fresh workspace; returns (O, Q, d).  uniform: no cu_new."""
    g = torch.Generator().manual_seed(seed)
    N = sum(new)
    Q = torch.randn((N, Hq, cache.D), generator=g).bfloat16().cuda() if Q is None else Q
    Lk = max(1, max(cache.lengths)) if Lk is None else Lk
    Lq = max(1, max(new)) if Lq is None else Lq
    p = l2a.params(len(new), Lq, Lk, Hq, cache.Hkv, cache.D, W, flags=flags, softmax_scale=scale)
    cu = None if uniform else torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    nbytes = l2a.l2a_cache_workspace_bytes(p, cache.handle, N)
    ws = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    out = torch.full((N + 2, Hq, cache.D), float("nan"), dtype=torch.bfloat16, device="cuda")
    if O is not None:
        out[1:N + 1] = O
    l2a.l2a_cache_forward(p, cache.handle, Q, cu, N, d, out[1:N + 1], ws[:nbytes])
    torch.cuda.synchronize()
    assert N == 0 or l2a.l2a_workspace_status(ws) == 0
    assert bool((ws[nbytes:] == 0xA5).all()), "wrote behind the workspace"
    assert bool(out[0].isnan().all()) and bool(out[N + 1].isnan().all()), "wrote outside O"
    return out[1:N + 1], Q


def routed(N, density, seed):
    g = torch.Generator().manual_seed(seed + 77)
    return (torch.rand(N, generator=g) < density).to(torch.uint8).cuda()
