"""The weights of cached keys in 64 bits, apart from the package, and the bound of their error.

A weight is exp(s) / sum exp(s') with scores in fp32: a score of D products is off by at most D 2^-24 sum |q_i k_i| scale, its product with
log2(e) and the subtraction by a rounding each, 2^-23 of the largest |s| together; numerator and denominator: twice that.  The exponentials are
off by 2^-22 each, sums of n positive terms by n 2^-24 at most.  Sums are made of partial sums (64 terms of a tile and lane, then the tiles), so
n is keys / 64 + 300 and rows / 64 + 300.  So each row's weights are off by at most
  2 (D 2^-24 A + 2^-22 A) + 2^-20 + (keys / 64 + rows / 64 + 600) 2^-24  of themselves,  A = max over keys of sum |q_i k_i| scale,
The old weight is added to for every 512 rows of a KV head (four blocks of 128 whose sums are made apart), with a rounding each time: at most
ceil(rows / 512) 2^-24 of the new weight, since all summands are positive."""
import math

import numpy as np
import torch

from paper_2603_17484_b200 import l2a


def weights(cache, Q, new, d, scale=None):
    """(increments, bounds of their error) of every sequence, [length, Hkv] in 64 bits."""
    N, Hq, D = Q.shape
    G = Hq // cache.Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, t = [], 0
    for b, n in enumerate(new):
        length = cache.lengths[b]
        inc = torch.zeros((length, cache.Hkv), dtype=torch.float64, device="cuda")
        off = torch.zeros_like(inc)
        pos = torch.arange(length - n, length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")[None]
        rows = int(d[t:t + n].sum()) * G if n else 0
        counts = d[t:t + n].double()[:, None]
        for h in range(Hq if length and n else 0):
            K = cache.K[b][:, h // G]
            q = Q[t:t + n, h].double()
            s = (q @ K.T * scale).masked_fill(j > pos, -math.inf)
            w = torch.exp(s - s.amax(1, keepdim=True).clamp(min=-1e300))
            w = w * (j <= pos)
            w = counts * w / w.sum(1, keepdim=True).clamp(min=1e-300)
            A = ((q.abs() @ K.abs().T * scale) * (j <= pos)).amax(1, keepdim=True)
            f = 2 * (D * 2.0 ** -24 + 2.0 ** -22) * A + 2.0 ** -20 + (length / 64 + rows / 64 + 600) * 2.0 ** -24
            inc[:, h // G] += w.sum(0)
            off[:, h // G] += (f * w).sum(0)
        out.append((inc, off))
        t += n
    return out


def weigh(cache, Hq, new, d, Q=None, seed=0, Lk=None, Lq=None, uniform=False, scale=0.0, calls=1, extra=0):
    """Calls on a fresh workspace and a pool of random weights (NaN where the new tokens' are to be); checks the result against weights()
    and that nothing else changed.  extra: rows of the token axis behind the last sequence.  Returns the pool."""
    g = torch.Generator().manual_seed(seed)
    N = sum(new)
    Q = torch.randn((N + extra, Hq, cache.D), generator=g).bfloat16().cuda() if Q is None else Q
    Lk = max(1, max(cache.lengths)) if Lk is None else Lk
    Lq = max(1, max(new)) if Lq is None else Lq
    page = cache.page
    n_pages = cache.poolK.shape[0]
    pool = (torch.rand((n_pages, cache.Hkv, page), generator=g) * 1e-3).cuda()
    slots = []
    for b, n in enumerate(new):
        j = torch.arange(cache.lengths[b], device="cuda")
        at = cache.table[b, j // page].long()
        slots.append((at, j % page))
        if n:
            pool[at[-n:], :, (j % page)[-n:]] = float("nan")
    before = pool.clone()
    p = l2a.params(len(new), Lq, Lk, Hq, cache.Hkv, cache.D, 5, softmax_scale=scale, q_stride=(0, Q.stride(0)))
    cu = None if uniform else torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    nbytes = l2a.l2a_cache_weigh_workspace_bytes(p, cache.handle, N + extra)
    ws = torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    for _ in range(calls):
        l2a.l2a_cache_weigh(p, cache.handle, Q, cu, N + extra, d, pool, ws[:nbytes])
    torch.cuda.synchronize()
    assert l2a.l2a_workspace_status(ws) == 0
    assert bool((ws[nbytes:] == 0xA5).all()), "wrote behind the workspace"
    count = torch.ones(N + extra, device="cuda") if d is None else d
    touched = torch.zeros_like(pool, dtype=torch.bool)
    for b, (inc, off) in enumerate(weights(cache, Q[:N], new, count[:N], scale or None)):
        at, slot = slots[b]
        n = new[b]
        if n == 0:
            continue
        old = before[at, :, slot].double()
        old[len(old) - n:] = 0
        # (the new tokens of a later call of the same are new again)
        times = torch.full((len(old), 1), float(calls), device="cuda", dtype=torch.float64)
        times[len(old) - n:] = 1
        want, got = old + times * inc, pool[at, :, slot].double()
        groups = max(1, math.ceil(int(count[sum(new[:b]):sum(new[:b + 1])].sum()) * (Hq // cache.Hkv) / 512))
        bound = times * off + times * groups * 2.0 ** -24 * want + 1e-36
        err = (got - want).abs()
        assert torch.isfinite(got).all(), f"sequence {b}: not finite"
        assert bool((err <= bound).all()), f"sequence {b}: {float((err / bound).max()):.3f} times the bound"
        touched[at[len(at) - n:], :, slot[len(at) - n:]] = True
        t = sum(new[:b])
        some = count[t:t + n].nonzero()
        hi = cache.lengths[b] - n + int(some.max()) if len(some) else -1
        if hi >= 0:
            touched[at[:hi + 1], :, slot[:hi + 1]] = True
    assert torch.equal(pool[~touched].view(torch.int32), before[~touched].view(torch.int32)), "a slot that no token has was touched"
    return pool
