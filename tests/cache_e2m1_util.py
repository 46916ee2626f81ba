"""The 4-bit format of the paged cache written plainly in 64 bits and apart from the package, and a cache of random sequences in it (or
in one of the other two) on the GPU.  What is computed from the cache has the tolerances of tests/cache_util.py."""
import numpy as np
import torch

from paper_2603_17484_b200 import l2a
from tests.cache_util import CODE_VALUES, Cache

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def nearest(y, table):
    """Index of the nearest entry of an ascending table, a tie to the even index; the last one above all."""
    hi = np.clip(np.searchsorted(table, y), 1, len(table) - 1)
    lo = hi - 1
    with np.errstate(invalid="ignore"):
        down, up = y - table[lo], table[hi] - y
    return np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)


def quantise4(rows):
    """(codes [..., D / 2], scales [..., D / 16], exponents + 127 [...]) of rows [..., D] given in 64 bits."""
    mag, negative = np.abs(rows), np.signbit(rows)
    fine = np.isfinite(mag)
    mag = np.where(fine, mag, 0.0)
    top = mag.max(-1)
    e = np.zeros(top.shape)
    some = top > 0
    f, x = np.frexp(top[some] / 2688.0)
    e[some] = np.maximum(np.where(np.ldexp(2688.0, x - 1) >= top[some], x - 1, x), -126)
    y = (mag / np.exp2(e)[..., None]).reshape(*mag.shape[:-1], mag.shape[-1] // 16, 16)
    s = nearest(y.max(-1) / 6, CODE_VALUES[:127])
    v = CODE_VALUES[s][..., None]
    code = nearest(np.where(v > 0, y / np.where(v > 0, v, 1.0), 0.0), MAGNITUDES).reshape(mag.shape) + 8 * negative
    lost = ~fine.reshape(*mag.shape[:-1], mag.shape[-1] // 16, 16).all(-1)
    s = np.where(lost, 0x7f, s)
    code = np.where(np.repeat(lost, 16, -1), 0, code)
    return (code[..., ::2] | code[..., 1::2] << 4).astype(np.uint8), s.astype(np.uint8), (e + 127).astype(np.uint8)


def decoded4(codes, scales, exponents):
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    return v * np.repeat(CODE_VALUES[scales], 16, -1) * np.exp2(exponents.astype(np.float64) - 127)[..., None]


class Cache4:
    """Sequences of given lengths in a shuffled pool, the fields of tests.cache_util.Cache.  Slots without a token hold NaN, table entries
    without a page a number that is none."""

    def __init__(self, page, Hkv, D, lengths, seed, per=None, interleaved=False, k_scale=1.0, v_scale=1.0, rows=None, spread=0.5):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.page, self.Hkv, self.D, self.lengths = "e2m1", page, Hkv, D, list(lengths)
        B = len(lengths)
        need = [-(-n // page) for n in lengths]
        per = max(1, max(need)) if per is None else per
        n_pages = sum(need) + 2
        order = torch.randperm(n_pages, generator=g)
        table = torch.randint(-(1 << 31), -1, (B, per), generator=g, dtype=torch.int64)
        table[:, ::2] = (1 << 31) - 1 - torch.arange(per)[::2]
        codes = torch.full((2, n_pages, Hkv, page, D // 2), 0x77, dtype=torch.uint8)
        exponents = torch.full((2, n_pages, Hkv, page), 255, dtype=torch.uint8)
        blocks = torch.full((2, n_pages, Hkv, page, D // 16), 0x7f, dtype=torch.uint8)
        true = [[], []]
        at = 0
        for b, n in enumerate(lengths):
            pages = order[at:at + need[b]]
            at += need[b]
            table[b, :need[b]] = pages
            j = torch.arange(n)
            for which, factor in ((0, k_scale), (1, v_scale)):
                x = (torch.randn((n, Hkv, D), generator=g) * factor * torch.exp(spread * torch.randn((n, Hkv, 1), generator=g))).bfloat16()
                if rows is not None:
                    x = rows(which, b, x)
                q, s, e = quantise4(x.double().numpy())
                codes[which][pages[j // page], :, j % page] = torch.from_numpy(q)
                blocks[which][pages[j // page], :, j % page] = torch.from_numpy(s)
                exponents[which][pages[j // page], :, j % page] = torch.from_numpy(e)
                true[which].append(torch.from_numpy(decoded4(q, s, e)))
        scales = torch.cat([exponents, blocks.flatten(3)], 3)
        if interleaved:                                  # K and V page by page in one allocation
            codes = codes.transpose(0, 1).contiguous().cuda().transpose(0, 1)
            scales = scales.transpose(0, 1).contiguous().cuda().transpose(0, 1)
        self.codes, self.scales = codes.cuda(), scales.cuda()
        self.poolK, self.poolV, self.ks, self.vs = *self.codes, *self.scales
        self.table, self.length = table.int().cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
        self.K, self.V = [x.cuda() for x in true[0]], [x.cuda() for x in true[1]]
        self.handle = self.handle_of(self.table, self.length)

    def handle_of(self, table, length):
        four = torch.float4_e2m1fn_x2
        return l2a.cache(self.poolK.view(four), self.poolV.view(four), table, length, k_scale=self.ks, v_scale=self.vs)


def make_cache(kind, page, Hkv, D, lengths, seed, **kw):
    return Cache4(page, Hkv, D, lengths, seed, **kw) if kind == "e2m1" else Cache(kind, page, Hkv, D, lengths, seed, **kw)
