"""Measurable cases of the operators that keep a long-lived paged key/value cache small.

Four operators on a pool of pages [pages, Hkv, page, D], of which every sequence has a table:

  store   writes a prompt's keys and values into a 4-bit cache and reads back what it stands for (append, then read)
  attend  attention of the new tokens over a 4-bit cache: the last W + 1 keys for all, all keys for the routed ones
  weigh   adds to a weight for every cached key what the routed new tokens' Global Attention gave it
  evict   keeps the first keys, the last ones and those of the highest weights in between, moved into other pages

A 4-bit row: D e2m1 codes, two a byte (the even element in the low half), an e4m3 scale for each 16 of them, a power of two for the
row.  Scales of a page and head: the rows' exponents + 127, [page], then the scales of their blocks, [page][D / 16].

Heads, head sizes, windows, context lengths and routed shares are those of the package's configurations and tests.
The plain forms are elementary torch operations in 32 bits on padded batches.
"""
from __future__ import annotations

import math
import random

import torch

own = False

E4M3_MAX, E2M1_MAX = 448.0, 6.0


def _case(name, kind, cache, B, new, ctx, ragged, page, Hq, Hkv, D, W, density=0.0, keep=0.0):
    c = {"kind": kind, "cache": cache, "B": B, "new": new, "ctx": ctx, "ragged": ragged, "page": page, "Hq": Hq,
         "Hkv": Hkv, "D": D, "W": W, "density": density, "keep": keep}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # ---- store: the latency of a sequence's first token
        _case("store_1_token", "store", "e2m1", 1, 1, 1, False, 64, 28, 4, 128, 4096),
        # short prompts of a batch, ragged, small heads in small pages
        _case("store_32_of_300", "store", "e2m1", 32, 300, 300, True, 16, 12, 2, 64, 128),
        # one long prompt
        _case("store_1_of_24k", "store", "e2m1", 1, 23999, 23999, False, 64, 32, 8, 128, 4096),
        # ---- attend: one token of a single user, routed
        _case("decode_1_of_9k", "attend", "e2m1", 1, 1, 9001, False, 64, 28, 4, 128, 4096, 1.0),
        # a serving batch of ragged contexts in small pages, one token in four routed
        _case("decode_32_of_8k", "attend", "e2m1", 32, 1, 8000, True, 16, 32, 8, 128, 4096, 0.25),
        # a large batch over long contexts, what 4 bits are for
        _case("decode_16_of_128k", "attend", "e2m1", 16, 1, 131072, False, 64, 32, 8, 128, 4096, 0.25),
        # chunks of several prompts of mixed lengths in one call
        _case("chunks_6_of_16k", "attend", "e2m1", 6, 500, 16384, True, 128, 28, 4, 128, 4096, 0.2),
        # the next 2000 tokens of a long prompt
        _case("chunk_2k_of_34k", "attend", "e2m1", 1, 2000, 34768, False, 64, 32, 8, 128, 4096, 0.2),
        # ---- weigh: the weights kept up to date with every decoded token of a batch
        _case("weigh_16_of_32k", "weigh", "e2m1", 16, 1, 32768, True, 64, 32, 8, 128, 4096, 0.5),
        # the last chunks of several prompts, whose attention says what of the prompt matters
        _case("weigh_chunks_4_of_16k", "weigh", "bf16", 4, 400, 16384, True, 64, 28, 4, 128, 4096, 0.3),
        # ---- evict: one user's cache back to half of it
        _case("evict_1_of_9k", "evict", "bf16", 1, 1, 9001, False, 64, 28, 4, 128, 1000, keep=0.5),
        # a batch's long caches at once
        _case("evict_16_of_32k", "evict", "e2m1", 16, 1, 32768, True, 64, 32, 8, 128, 4096, keep=0.4),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    Hq, Hkv, D = rng.choice([(28, 4, 128), (32, 8, 128), (28, 4, 128), (32, 8, 128), (4, 4, 64), (12, 2, 64), (8, 1, 128)])
    W = rng.choice([128, 1000, 4096, 4096])
    page = rng.choice([16, 32, 64, 128])
    kind = rng.choice(["store", "decode", "decode", "chunk", "chunk", "weigh", "weigh_chunk", "evict"])
    cache = rng.choice(["e2m1", "e4m3", "bf16"])
    density = rng.choice([0.05, 0.1, 0.2, 0.2, 0.3, 0.5, 1.0])
    if kind == "store":
        B = size(1, 32)
        new = size(1, 24000 // B)
        return _case(None, kind, "e2m1", B, new, new, True, page, Hq, Hkv, D, W)
    if kind == "evict":
        ctx = size(16, 65536)
        B = size(1, max(1, min(32, (1 << 19) // ctx)))
        return _case(None, kind, cache, B, 1, ctx, rng.random() < 0.7, page, Hq, Hkv, D, W, keep=rng.choice([0.1, 0.25, 0.5, 0.9]))
    if kind in ("decode", "weigh"):
        ctx = size(1, 131072)
        B = size(1, max(1, min(64, (1 << 21 if kind == "decode" else 1 << 19) // ctx)))
        ragged = rng.random() < 0.7
        if kind == "decode":
            return _case(None, "attend", "e2m1", B, 1, ctx, ragged, page, Hq, Hkv, D, W, rng.choice([0.0, density]))
        return _case(None, "weigh", cache, B, 1, ctx, ragged, page, Hq, Hkv, D, W, density)
    ctx = size(64, 65536)
    new = size(2, min(4096, ctx, 2_000_000_000 // (Hq * ctx)))
    B = size(1, max(1, min(8, 2_000_000_000 // (Hq * ctx * new))))
    if kind == "chunk":
        return _case(None, "attend", "e2m1", B, new, ctx, rng.random() < 0.7, page, Hq, Hkv, D, W, density)
    return _case(None, "weigh", cache, B, new, ctx, rng.random() < 0.7, page, Hq, Hkv, D, W, density)


# ----------------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """(tokens, new tokens) of every sequence: a function of the case alone.  The first has the most of both."""
    B, new, ctx = case["B"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [ctx] * B, [new] * B
    r = random.Random(B * 1000003 + new * 101 + ctx)
    n = [new] + [max(1, round(new * r.random())) for _ in range(B - 1)]
    if case["kind"] == "store":
        return n, n
    length = [ctx] + [max(n[i], round(ctx * 8 ** -r.random())) for i in range(1, B)]
    return length, n


def _kept(case):
    """What an eviction keeps: (tokens of every sequence, first ones, last ones)."""
    length, _ = _lengths(case)
    recent = min(case["W"], case["ctx"] // 4)
    return [max(1, round(x * case["keep"])) for x in length], 4, recent


def _routed(case, N):
    return 0 if case["density"] == 0 else max(1, round(case["density"] * N))


def _quantised8(x):
    """e4m3 codes and biased exponents of bf16 rows: the least power of two 2^e with max |x| <= 448 * 2^e."""
    mant, ex = torch.frexp(x.abs().amax(-1).float())
    e = torch.where(mant > 0, ex - 9 + (mant > 0.875).int(), 0).clamp(-126, 127)
    inv = ((127 - e) << 23).view(torch.float32)
    return (x.float() * inv.unsqueeze(-1)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _quantised4(x):
    """Rows in 4 bits: codes [..., D / 2], scales of 16 (as e4m3's bytes) [..., D / 16], biased exponents [...].  The nearest of
    0, 1/2, 1, 3/2, 2, 3, 4, 6 is the number of borders between them that a value is past; a value on a border goes to the even code."""
    x = x.float()
    mant, ex = torch.frexp(x.abs().amax(-1))
    e = torch.where(mant > 0, ex - 12 + (mant > 0.65625).int(), 0).clamp(-126, 127)      # 6 * 448 = 0.65625 * 2^12
    x = (x * ((127 - e) << 23).view(torch.float32).unsqueeze(-1)).unflatten(-1, (-1, 16))
    s = (x.abs().amax(-1) / E2M1_MAX).to(torch.float8_e4m3fn)
    y = torch.where(s.float().unsqueeze(-1) > 0, x.abs() / s.float().unsqueeze(-1), 0.0)
    code = (y > 0.25).byte() + (y >= 0.75).byte() + (y > 1.25).byte() + (y >= 1.75).byte() + (y > 2.5).byte() + (y >= 3.5).byte() + (y > 5.0).byte()
    code = (code + 8 * torch.signbit(x).byte()).flatten(-2)
    return code[..., ::2] | code[..., 1::2] << 4, s.view(torch.uint8), (e + 127).to(torch.uint8)


def _with_scales(e, s):
    """Exponents [pages, Hkv, page] and scales [pages, Hkv, page, D / 16] as a page keeps them."""
    return torch.cat([e, s.flatten(2)], 2).contiguous()


def prepare(case, seed):
    B, Hq, Hkv, D, page, kind = (case[k] for k in ("B", "Hq", "Hkv", "D", "page", "kind"))
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    length, n = _lengths(case)
    N, most, most_new = sum(n), max(length), max(n)
    per = -(-most // page)
    need = sum(-(-x // page) for x in length)
    pool = need + 3                                          # a pool has pages of nobody
    perm = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)

    def table_of(lengths, entries):
        rows = torch.tensor([-(-x // page) for x in lengths], device="cuda")
        i = torch.arange(entries, device="cuda")
        at = (rows.cumsum(0) - rows)[:, None] + i
        return torch.where(i < rows[:, None], perm[at.clamp(max=pool - 1)], -1).to(torch.int32)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    # keys have channels of unequal size, values tokens of unequal size
    chan = torch.exp(0.4 * torch.randn((Hkv, 1, D), generator=g, device="cuda")).to(torch.bfloat16)

    def rows(values):
        x = normal(pool, Hkv, page, D)
        if values:
            return x.mul_(torch.exp(0.3 * torch.randn((pool, Hkv, page, 1), generator=g, device="cuda")).to(torch.bfloat16))
        return x.mul_(chan)

    s = {"case": dict(case), "table": table_of(length, per), "lengths": torch.tensor(length, dtype=torch.int32, device="cuda"),
         "cu": torch.tensor([sum(n[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda"), "N": N,
         "most": most, "most_new": most_new}
    # slots that hold no token hold whatever was there: NaN
    pos = torch.arange(per * page, device="cuda")
    ok = (pos[None, :] < s["lengths"][:, None]).view(B, per, page)
    live = torch.zeros((pool, page), dtype=torch.bool, device="cuda")
    live[s["table"].long().clamp(min=0)[ok.any(-1)]] = ok[ok.any(-1)]
    dead = ~live
    for name in ("K", "V"):
        if kind == "store":
            s[name] = torch.zeros((pool, Hkv, page, D // 2), dtype=torch.uint8, device="cuda")
            s["e" + name] = torch.zeros((pool, Hkv, page * (1 + D // 16)), dtype=torch.uint8, device="cuda")
            continue
        x = rows(name == "V")
        if case["cache"] == "e4m3":
            x, e = _quantised8(x)
            x.view(torch.uint8).masked_fill_(dead[:, None, :, None], 0x7f)
            s["e" + name] = e.masked_fill_(dead[:, None, :], 255)
        elif case["cache"] == "e2m1":
            x, t, e = _quantised4(x)
            s["e" + name] = _with_scales(e.masked_fill_(dead[:, None, :], 255), t.masked_fill_(dead[:, None, :, None], 0x7f))
        else:
            x.masked_fill_(dead[:, None, :, None], float("nan"))
        s[name] = x
    if kind == "store":
        s["newK"] = normal(N, Hkv, D).mul_(chan[:, 0])
        s["newV"] = normal(N, Hkv, D)
        s["outK"] = torch.empty((B, most, Hkv, D), dtype=torch.bfloat16, device="cuda")
        s["outV"] = torch.empty_like(s["outK"])
    if kind in ("attend", "weigh"):
        s["Q"] = normal(N, Hq, D)
        d = torch.zeros(N, dtype=torch.uint8, device="cuda")
        d[torch.randperm(N, generator=g, device="cuda")[:_routed(case, N)]] = 1
        s["d"] = d
        s["O"] = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda")
    if kind in ("weigh", "evict"):
        # weights are sums of many small ones with a few large, here those of one routed token; keys that none has seen have none
        w = torch.exp(1.5 * torch.randn((pool, Hkv, page), generator=g, device="cuda")) * (Hq / Hkv / case["ctx"])
        s["w"] = w.masked_fill_(torch.rand((pool, Hkv, page), generator=g, device="cuda") < 0.1, 0.0)
    if kind == "evict":
        keep, s["sinks"], s["recent"] = _kept(case)
        s["most_kept"] = max(keep)
        s["keep"] = torch.tensor(keep, dtype=torch.int32, device="cuda")
        perm = perm.flip(0)                                  # of a pool of their own, as large
        s["table2"] = table_of(keep, -(-max(keep) // page))
        for name in ("K", "V", "eK", "eV", "w"):
            if name in s:
                s[name + "2"] = torch.zeros_like(s[name])
        s["lengths2"] = torch.zeros_like(s["lengths"])
        s["kept"] = torch.zeros((B, Hkv, max(keep)), dtype=torch.int32, device="cuda")
    if own:                                                  # the descriptions and the workspace that a program keeps
        s.update(_handles(s))
    return s


def _handles(s):
    from paper_2603_17484_b200 import l2a

    c = s["case"]

    def cache(suffix):
        K, V = s["K" + suffix], s["V" + suffix]
        if c["cache"] == "e2m1":
            K, V = K.view(torch.float4_e2m1fn_x2), V.view(torch.float4_e2m1fn_x2)
        return l2a.cache(K, V, s["table" + suffix], s["lengths" + suffix], k_scale=s.get("eK" + suffix), v_scale=s.get("eV" + suffix))

    Lq = s["most_kept"] if c["kind"] == "evict" else s["most_new"]
    p = l2a.params(c["B"], Lq, s["most"], c["Hq"], c["Hkv"], c["D"], c["W"])
    h = {"l2a": l2a, "p": p, "cache": cache("")}
    if c["kind"] == "evict":
        h["cache2"] = cache("2")
        size = l2a.l2a_cache_evict_workspace_bytes(p, h["cache"])
    elif c["kind"] == "weigh":
        size = l2a.l2a_cache_weigh_workspace_bytes(p, h["cache"], s["N"])
    else:
        size = l2a.l2a_cache_workspace_bytes(p, h["cache"], s["N"]) if c["kind"] == "attend" else 256
    h["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return h


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"store": _plain_store, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[kind](s)
    l2a = s["l2a"]
    if kind == "store":
        l2a.l2a_cache_append(s["p"], s["cache"], s["newK"], s["newV"], s["cu"], s["N"])
        l2a.l2a_cache_read(s["p"], s["cache"], None, s["outK"], s["outV"])
        return {"K": s["outK"], "V": s["outV"]}
    if kind == "attend":
        l2a.l2a_cache_forward(s["p"], s["cache"], s["Q"], s["cu"], s["N"], s["d"], s["O"], s["ws"])
        return s["O"]
    if kind == "weigh":
        l2a.l2a_cache_weigh(s["p"], s["cache"], s["Q"], s["cu"], s["N"], s["d"], s["w"], s["ws"])
        return s["w"]
    l2a.l2a_cache_evict(s["p"], s["cache"], s["w"], s["keep"], s["sinks"], s["recent"], s["cache2"], s["w2"], s["lengths2"],
                        s["kept"], s["ws"])
    return _moved(s)


def _moved(s):
    """What an eviction leaves.  It computes no values: 4-bit rows come as the bytes that were moved."""
    return {k: s[k] for k in ("K2", "V2", "eK2", "eV2", "w2", "lengths2", "kept") if k in s}


# ---------------------------------------------------------------------------------------------------- plain forms
def _positions(s):
    """Sequence and position of every new token."""
    t = torch.arange(s["N"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    return b, s["lengths"][b] - s["cu"][b + 1] + t


def _plain_values4(codes, scales, page, D):
    """What 4-bit rows [..., page, D / 2] with their scales [..., page * (1 + D / 16)] stand for."""
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    x = torch.stack([value[(codes & 15).int()], value[(codes >> 4).int()]], -1).flatten(-2).unflatten(-1, (-1, 16))
    e, t = scales[..., :page], scales[..., page:].contiguous().view(torch.float8_e4m3fn).unflatten(-1, (page, -1))
    return ((x * t.float().unsqueeze(-1)).flatten(-2)) * (e.int() << 23).view(torch.float32).unsqueeze(-1)


def _plain_dense(s, name):
    """[B, Hkv, keys, D] in 32 bits, zeros behind a sequence's end."""
    c = s["case"]
    at = s["table"].long().clamp(min=0)
    if c["cache"] == "e2m1":
        x = _plain_values4(s[name][at], s["e" + name][at], c["page"], c["D"])
    else:
        x = s[name][at].float()
        if "e" + name in s:
            x = x * (s["e" + name][at].int() << 23).view(torch.float32).unsqueeze(-1)
    x = x.permute(0, 2, 1, 3, 4).reshape(c["B"], c["Hkv"], -1, c["D"])[:, :, :s["most"]]
    j = torch.arange(s["most"], device="cuda")
    return torch.where((j < s["lengths"][:, None])[:, None, :, None], x, 0.0)


def _plain_store(s):
    c = s["case"]
    page, D = c["page"], c["D"]
    b, pos = _positions(s)
    at, slot = s["table"][b, pos // page].long(), (pos % page).long()
    for name in ("K", "V"):
        codes, t, e = _quantised4(s["new" + name])
        s[name][at, :, slot] = codes
        s["e" + name][at, :, slot] = e
        s["e" + name][:, :, page:].unflatten(2, (page, D // 16))[at, :, slot] = t
    return {name: _plain_dense(s, name).transpose(1, 2).to(torch.bfloat16).contiguous() for name in ("K", "V")}


def _plain_scores(s):
    """Scores [B, Hkv, new, G, keys] of the new tokens, a padded batch, -inf behind each one's position; and sequence, index and
    position of every new token, positions [B, new] (-1: none)."""
    c = s["case"]
    B, Hq, Hkv, D, L = c["B"], c["Hq"], c["Hkv"], c["D"], s["most_new"]
    b, pos = _positions(s)
    i = torch.arange(s["N"], device="cuda") - s["cu"][b]
    Q = torch.zeros((B, L, Hq, D), device="cuda")
    Q[b, i] = s["Q"].float()
    p = torch.full((B, L), -1, dtype=torch.int32, device="cuda")
    p[b, i] = pos
    Q = Q.view(B, L, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    S = (Q @ _plain_dense(s, "K").transpose(2, 3)).mul_(D ** -0.5).view(B, Hkv, L, Hq // Hkv, -1)
    j = torch.arange(s["most"], device="cuda", dtype=torch.int32)
    S.masked_fill_(~(j <= p[:, :, None])[:, None, :, None, :], -math.inf)
    d = torch.zeros((B, L), device="cuda")
    d[b, i] = s["d"].float()
    return S, b, i, p, d


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hkv, D, L = c["B"], c["Hq"], c["Hkv"], c["D"], s["most_new"]
    S, b, i, p, d = _plain_scores(s)
    V = _plain_dense(s, "V")
    j = torch.arange(s["most"], device="cuda", dtype=torch.int32)
    near = (j >= p[:, :, None] - c["W"])[:, None, :, None, :]
    S.sub_(S.amax(-1, keepdim=True).clamp(min=-1e30))
    glb = S.exp()
    a = (glb.view(B, Hkv, -1, glb.shape[-1]) @ V).view(B, Hkv, L, -1, D) / glb.sum(-1, keepdim=True).clamp(min=1e-38)
    del glb
    S.masked_fill_(~near, -math.inf)
    S.sub_(S.amax(-1, keepdim=True).clamp(min=-1e30))
    loc = S.exp_()
    o = (loc.view(B, Hkv, -1, loc.shape[-1]) @ V).view(B, Hkv, L, -1, D) / loc.sum(-1, keepdim=True).clamp(min=1e-38)
    o = o + d[:, None, :, None, None] * a
    return o.permute(0, 2, 1, 3, 4).reshape(B, L, Hq, D)[b, i].to(torch.bfloat16)


def _plain_weigh(s):
    c = s["case"]
    S, b, i, p, d = _plain_scores(s)
    S.sub_(S.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    S.mul_((d[:, None, :, None, None] / S.sum(-1, keepdim=True).clamp(min=1e-38)))
    add = S.sum((2, 3))                                      # [B, Hkv, keys]
    j = torch.arange(s["most"], device="cuda")
    at, slot = s["table"].long().clamp(min=0)[:, j // c["page"]], (j % c["page"]).expand(c["B"], -1)
    ahead = s["lengths"] - (s["cu"][1:] - s["cu"][:-1])      # tokens before the new ones: those have weights already
    old = torch.where((j < ahead[:, None])[..., None], s["w"][at, :, slot], 0.0)
    ok = j < s["lengths"][:, None]
    s["w"].transpose(1, 2)[at[ok], slot[ok]] = (old + add.transpose(1, 2))[ok]
    return s["w"]


def _plain_evict(s):
    c = s["case"]
    page = c["page"]
    j = torch.arange(s["most"], device="cuda")
    at, slot = s["table"].long().clamp(min=0)[:, j // page], (j % page).expand(c["B"], -1)
    w = s["w"][at, :, slot].transpose(1, 2)                  # [B, Hkv, keys]
    n = s["lengths"][:, None]
    kept = torch.minimum(s["keep"][:, None], n)
    recent = torch.minimum(torch.full_like(kept, s["recent"]), kept)
    sinks = torch.minimum(torch.full_like(kept, s["sinks"]), kept - recent)
    always = ((j < sinks) | (j >= n - recent)) & (j < n)
    w = torch.where(always[:, None], math.inf, torch.where((j < n)[:, None], w, -math.inf))
    order = w.sort(dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, j.expand_as(order))
    take = rank < kept[:, None]                              # [B, Hkv, keys]
    to = take.cumsum(-1) - 1
    s["kept"].fill_(-1)
    b, g, x = take.nonzero(as_tuple=True)
    to = to[b, g, x]
    s["kept"][b, g, to] = x.int()
    s["lengths2"].copy_(kept[:, 0])
    p1, i1, p2, i2 = s["table"][b, x // page].long(), x % page, s["table2"][b, to // page].long(), to % page
    s["w2"][p2, g, i2] = s["w"][p1, g, i1]
    for name in ("K", "V"):
        s[name + "2"].view(torch.uint8 if c["cache"] != "bf16" else torch.int16)[p2, g, i2] = \
            s[name].view(torch.uint8 if c["cache"] != "bf16" else torch.int16)[p1, g, i1]
        if c["cache"] == "e4m3":
            s["e" + name + "2"][p2, g, i2] = s["e" + name][p1, g, i1]
        elif c["cache"] == "e2m1":
            new, old = s["e" + name + "2"], s["e" + name]
            new[p2, g, i2] = old[p1, g, i1]
            shape = (page, c["D"] // 16)
            new[:, :, page:].unflatten(2, shape)[p2, g, i2] = old[:, :, page:].unflatten(2, shape)[p1, g, i1]
    return _moved(s)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _of_bits(c, exponent_bits, mantissa_bits, bias):
    """Values of small floats from their bits, without a sign."""
    mant, ex = c & ((1 << mantissa_bits) - 1), (c >> mantissa_bits) & ((1 << exponent_bits) - 1)
    whole = torch.where(ex > 0, mant + (1 << mantissa_bits), mant).double()
    return whole * torch.exp2((ex.clamp(min=1) - bias - mantissa_bits).double())


def _rounded(x, mantissa_bits, least, most):
    """To 1 + mantissa_bits significant bits, ties to even, no finer than at 2^least, at most `most`."""
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=least).double() - mantissa_bits)
    return (torch.round(x / step) * step).clamp(-most, most)


def _coded4(x):
    """What 4-bit rows stand for, all in 64 bits from the definition."""
    x = x.double()
    top = x.abs().amax(-1)
    mant, e = torch.frexp(top / (E2M1_MAX * E4M3_MAX))       # the least power of two not below: 2^(e - 1) for mant = 1/2
    e = torch.where(top > 0, e - (mant == 0.5).int(), 0).clamp(-126, 127).double()
    unit = torch.exp2(e)[..., None, None]
    x = x.unflatten(-1, (-1, 16)) / unit
    s = _rounded(x.abs().amax(-1, keepdim=True) / E2M1_MAX, 3, -6, E4M3_MAX)
    y = torch.where(s > 0, _rounded(x / torch.where(s > 0, s, 1.0), 1, 0, E2M1_MAX), 0.0)
    return (y * s * unit).flatten(-2)


def _sequence(s, name, b, length, g):
    """Keys or values of KV head g of sequence b, [length, D], in 64 bits."""
    c = s["case"]
    page, D = c["page"], c["D"]
    pages = s["table"][b, :-(-length // page)].long()
    x = s[name][pages, g]
    if c["cache"] == "bf16":
        x = x.double()
    else:
        e = s["e" + name][pages, g].int()
        if c["cache"] == "e4m3":
            u = x.view(torch.uint8).int()
            x = (1 - 2 * (u >> 7)) * _of_bits(u & 127, 4, 3, 7)
        else:
            u = torch.stack([x & 15, x >> 4], -1).flatten(-2).int()
            t = _of_bits(e[:, page:].reshape(-1, page, D // 16), 4, 3, 7).repeat_interleave(16, -1)
            x = (1 - 2 * (u >> 3)) * _of_bits(u & 7, 2, 1, 1) * t
        x = x * torch.exp2((e[:, :page] - 127).double()).unsqueeze(-1)
    return x.reshape(-1, D)[:length]


def exact(case, seed):
    s = prepare(case, seed)
    length, n = _lengths(case)
    B, page, D, Hkv, G = case["B"], case["page"], case["D"], case["Hkv"], case["Hq"] // case["Hkv"]
    if case["kind"] == "store":
        out = {name: torch.zeros((B, s["most"], Hkv, D), dtype=torch.float64, device="cuda") for name in ("K", "V")}
        for b in range(B):
            for name in ("K", "V"):
                out[name][b, :n[b]] = _coded4(s["new" + name][sum(n[:b]):sum(n[:b + 1])])
        return out
    if case["kind"] == "evict":
        return _exact_evict(case, s)
    O = torch.zeros((s["N"], case["Hq"], D), dtype=torch.float64, device="cuda")
    W = s["w"].double() if case["kind"] == "weigh" else None
    for b in range(B):
        rows = slice(sum(n[:b]), sum(n[:b + 1]))
        p = torch.arange(length[b] - n[b], length[b], device="cuda")[:, None]
        j = torch.arange(length[b], device="cuda")
        routed = s["d"][rows].double()
        at, slot = s["table"][b][j // page].long(), j % page
        for g in range(Hkv):
            K = _sequence(s, "K", b, length[b], g)
            V = _sequence(s, "V", b, length[b], g) if W is None else None
            weight = torch.where(j < length[b] - n[b], W[at, g, slot], 0.0) if W is not None else None
            for h in range(g * G, (g + 1) * G):
                w = torch.exp(s["Q"][rows, h].double() @ K.T / math.sqrt(D))
                w = w * (j <= p)
                if W is not None:
                    weight = weight + routed @ (w / w.sum(1, keepdim=True))
                    continue
                near = w * (j >= p - case["W"])
                O[rows, h] = near @ V / near.sum(1, keepdim=True) + routed[:, None] * (w @ V / w.sum(1, keepdim=True))
            if W is not None:
                W[at, g, slot] = weight
    return O if W is None else W


def _exact_evict(case, s):
    length, _ = _lengths(case)
    keep, sinks, recent = _kept(case)
    page, Hkv = case["page"], case["Hkv"]
    w2 = torch.zeros(s["w2"].shape, dtype=torch.float64, device="cuda")
    K2, V2 = (torch.zeros(s["K"].shape, dtype=torch.float64, device="cuda") for _ in range(2)) if case["cache"] != "e2m1" else (None, None)
    kept = torch.full(s["kept"].shape, -1, dtype=torch.int32, device="cuda")
    for b in range(case["B"]):
        n, m = length[b], min(length[b], keep[b])
        r = min(recent, m)
        f = min(sinks, m - r)
        j = torch.arange(n, device="cuda")
        at, slot = s["table"][b][j // page].long(), j % page
        to = torch.arange(m, device="cuda")
        at2, slot2 = s["table2"][b][to // page].long(), to % page
        for g in range(Hkv):
            middle = s["w"][at, g, slot].double()[f:n - r]
            best = torch.argsort(-middle, stable=True)[:m - r - f] + f
            x = torch.cat([j[:f], best.sort().values, j[n - r:]])
            kept[b, g, :m] = x.int()
            w2[at2, g, slot2] = s["w"][at[x], g, slot[x]].double()
            if K2 is not None:
                K2[at2, g, slot2] = s["K"][at[x], g, slot[x]].double()
                V2[at2, g, slot2] = s["V"][at[x], g, slot[x]].double()
    return {k: {"K2": K2, "V2": V2, "w2": w2, "kept": kept}.get(k) for k in _moved(s)}


# ---------------------------------------------------------------------------------------------------- work
def work(case):
    """Each key that some row sees is read once, each result written once; for a visible pair of a query row and a key two operations
    an element of a product, the pairs inside the window once for both attentions."""
    length, n = _lengths(case)
    N, Hq, Hkv, D, W = sum(n), case["Hq"], case["Hkv"], case["D"], case["W"]
    row = {"e2m1": D / 2 + D / 16 + 1, "e4m3": D + 1, "bf16": 2 * D}[case["cache"]]      # a key or a value as held
    if case["kind"] == "store":
        return {"bytes": 2.0 * N * Hkv * (2 * D + row) + 4.0 * case["B"] * max(length) * Hkv * D, "flops": 0.0}
    if case["kind"] == "evict":
        keep = [min(x, y) for x, y in zip(_kept(case)[0], length)]
        return {"bytes": Hkv * (4.0 * sum(length) + sum(keep) * (2 * (2 * row + 4.0) + 4.0)), "flops": 0.0}
    rho = _routed(case, N) / N
    keys = pairs = 0.0
    for total, new in zip(length, n):
        first = total - new
        some = 1 - (1 - rho) ** new                                          # the share of calls in which one is routed
        if case["kind"] == "weigh":
            keys += some * total
            pairs += rho * sum(range(first + 1, total + 1))
            continue
        window = total - max(0, first - W)
        keys += window + some * (total - window)
        for p in range(first, total):
            near = min(p, W) + 1
            pairs += near + rho * (p + 1 - near)
    if case["kind"] == "weigh":
        return {"bytes": keys * Hkv * (row + 8.0) + 2.0 * rho * N * Hq * D, "flops": 2.0 * D * Hq * pairs}
    return {"bytes": 2 * keys * Hkv * row + 4.0 * N * Hq * D, "flops": 4.0 * D * Hq * pairs}
