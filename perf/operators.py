"""Measurable cases of the operators that serve the L2A layer from a paged key/value cache.

Three operators, on a pool of pages [pages, Hkv, page, D] in bf16 or in 8 bits (e4m3 with a power-of-two scale for each
token and KV head), of which every sequence has a table:

  append  writes the keys and values of the new tokens of every sequence into its pages (and quantises them)
  read    reads the pages of every sequence back into dense bf16 tensors
  attend  attention of the new tokens over the cache: the last W + 1 keys for all, all keys for the routed ones,
          o = s + d * a; one new token per sequence (decode) as well as chunks of a prompt

Heads, head sizes, windows, context lengths and routed shares are those of the package's configurations and tests.
The plain forms are elementary torch operations in 32 bits on padded batches.
"""
from __future__ import annotations

import math
import random

import torch

own = False

E4M3_MAX = 448.0


def _case(name, kind, cache, B, new, ctx, ragged, page, Hq, Hkv, D, W, density=0.0):
    c = {"kind": kind, "cache": cache, "B": B, "new": new, "ctx": ctx, "ragged": ragged, "page": page, "Hq": Hq,
         "Hkv": Hkv, "D": D, "W": W, "density": density}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # ---- append: the latency of one token of one user
        _case("append_1_token", "append", "e4m3", 1, 1, 9001, False, 64, 28, 4, 128, 4096),
        # one token for every sequence of a serving batch, unquantised cache in small pages
        _case("append_32_tokens_bf16", "append", "bf16", 32, 1, 8000, True, 16, 32, 8, 128, 4096),
        # a prompt's chunk for a few sequences at once, ragged
        _case("append_chunks_8k", "append", "e4m3", 3, 8155, 16384, True, 64, 32, 8, 128, 4096),
        # ---- read: one prompt taken out of the cache (to be kept elsewhere, or recomputed from)
        _case("read_1_of_9k", "read", "e4m3", 1, 1, 9001, False, 16, 28, 4, 128, 4096),
        # a batch's caches, ragged
        _case("read_8_of_32k", "read", "e4m3", 8, 1, 32768, True, 64, 32, 8, 128, 4096),
        # ---- attend, one token per sequence: a single user, routed
        _case("decode_1_of_9k", "attend", "e4m3", 1, 1, 9001, False, 64, 28, 4, 128, 4096, 1.0),
        # a serving batch of ragged contexts over an unquantised cache in small pages, one token in four routed
        _case("decode_32_of_8k_bf16", "attend", "bf16", 32, 1, 8000, True, 16, 32, 8, 128, 4096, 0.25),
        # a large batch over long contexts, a quarter of the tokens routed
        _case("decode_16_of_128k", "attend", "e4m3", 16, 1, 131072, False, 64, 32, 8, 128, 4096, 0.25),
        # a few drafted tokens of every sequence to be verified at once
        _case("verify_8x5_of_32k", "attend", "e4m3", 8, 5, 32768, True, 32, 28, 4, 128, 4096, 0.2),
        # small heads, small window, a short chunk
        _case("chunk_200_of_2k_bf16", "attend", "bf16", 1, 200, 2000, False, 16, 12, 2, 64, 128, 0.2),
        # chunks of several prompts of mixed lengths in one call
        _case("chunks_6_of_16k", "attend", "e4m3", 6, 500, 16384, True, 128, 28, 4, 128, 4096, 0.2),
        # the next 2000 tokens of a long prompt
        _case("chunk_2k_of_34k", "attend", "e4m3", 1, 2000, 34768, False, 64, 32, 8, 128, 4096, 0.2),
    ]


def draw(rng):
    """One more case of the same ranges."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    Hq, Hkv, D = rng.choice([(28, 4, 128), (32, 8, 128), (28, 4, 128), (32, 8, 128), (4, 4, 64), (12, 2, 64), (8, 1, 128)])
    W = rng.choice([128, 1000, 4096, 4096])
    cache = rng.choice(["e4m3", "e4m3", "bf16"])
    page = rng.choice([16, 32, 64, 128])
    kind = rng.choice(["append", "read", "decode", "decode", "chunk", "chunk"])
    density = rng.choice([0.05, 0.1, 0.2, 0.2, 0.3, 0.5, 1.0])
    if kind == "append":
        B = size(1, 32)
        new = size(1, 24000 // B)
        return _case(None, kind, cache, B, new, min(new + size(1, 16384), 40000), True, page, Hq, Hkv, D, W)
    if kind == "read":
        B = size(1, 16)
        return _case(None, kind, cache, B, 1, size(1, (1 << 18) // B), rng.random() < 0.7, page, Hq, Hkv, D, W)
    if kind == "decode":
        ctx = size(1, 131072)
        B = size(1, min(64, (1 << 21) // ctx))
        return _case(None, "attend", cache, B, 1, ctx, rng.random() < 0.7, page, Hq, Hkv, D, W, rng.choice([0.0, density]))
    ctx = size(64, 65536)
    new = size(2, min(4096, ctx, 2_000_000_000 // (Hq * ctx)))
    B = size(1, max(1, min(8, 2_000_000_000 // (Hq * ctx * new))))
    return _case(None, "attend", cache, B, new, ctx, rng.random() < 0.7, page, Hq, Hkv, D, W, density)


# ----------------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """(tokens, new tokens) of every sequence: a function of the case alone.  The first has the most of both."""
    B, new, ctx = case["B"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [ctx] * B, [new] * B
    r = random.Random(B * 1000003 + new * 101 + ctx)
    n = [new] + [max(1, round(new * r.random())) for _ in range(B - 1)]
    length = [ctx] + [max(n[i], round(ctx * 8 ** -r.random())) for i in range(1, B)]
    return length, n


def _quantised(x):
    """e4m3 codes and biased exponents of bf16 rows, the formula of the cache: the least power of two 2^e with
    max |x| <= 448 * 2^e."""
    mant, ex = torch.frexp(x.abs().amax(-1).float())
    e = torch.where(mant > 0, ex - 9 + (mant > 0.875).int(), 0).clamp(-126, 127)
    inv = ((127 - e) << 23).view(torch.float32)
    return (x.float() * inv.unsqueeze(-1)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    B, Hq, Hkv, D, page, kind = (case[k] for k in ("B", "Hq", "Hkv", "D", "page", "kind"))
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    length, n = _lengths(case)
    N, most, most_new = sum(n), max(length), max(n)
    per = -(-most // page)                                   # pages of the longest sequence, columns of the table
    need = sum(-(-x // page) for x in length)
    pool = need + 3                                          # a pool has pages of nobody
    perm = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, per), -1, dtype=torch.int32)
    used, at = perm.cpu(), 0
    for b in range(B):
        k = -(-length[b] // page)
        table[b, :k] = used[at:at + k]
        at += k

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    # keys have channels of unequal size, values tokens of unequal size
    chan = torch.exp(0.4 * torch.randn((Hkv, 1, D), generator=g, device="cuda")).to(torch.bfloat16)

    def rows(values):
        x = normal(pool, Hkv, page, D)
        if values:
            return x.mul_(torch.exp(0.3 * torch.randn((pool, Hkv, page, 1), generator=g, device="cuda")).to(torch.bfloat16))
        return x.mul_(chan)

    s = {"case": dict(case), "table": table.cuda(), "lengths": torch.tensor(length, dtype=torch.int32, device="cuda"),
         "cu": torch.tensor([sum(n[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda"), "N": N,
         "most": most, "most_new": most_new}
    # slots that hold no token: zeros where the pool itself is the result, else whatever was there
    live = torch.zeros((pool, page), dtype=torch.bool, device="cuda")
    pos = torch.arange(per * page, device="cuda")
    ok = (pos[None, :] < s["lengths"][:, None]).view(B, per, page)
    live[s["table"].long().clamp(min=0)[ok.any(-1)]] = ok[ok.any(-1)]
    dead = ~live
    for name in ("K", "V"):
        x = rows(name == "V")
        if case["cache"] == "e4m3":
            x, e = _quantised(x)
            x.view(torch.uint8).masked_fill_(dead[:, None, :, None], 0 if kind == "append" else 0x7f)
            e.masked_fill_(dead[:, None, :], 0 if kind == "append" else 255)
            s["e" + name] = e
        else:
            x.masked_fill_(dead[:, None, :, None], 0.0 if kind == "append" else float("nan"))
        s[name] = x
    if kind == "append":
        s["newK"] = normal(N, Hkv, D).mul_(chan[:, 0])
        s["newV"] = normal(N, Hkv, D)
    elif kind == "read":
        s["outK"] = torch.empty((B, most, Hkv, D), dtype=torch.bfloat16, device="cuda")
        s["outV"] = torch.empty_like(s["outK"])
    else:
        s["Q"] = normal(N, Hq, D)
        d = torch.zeros(N, dtype=torch.uint8, device="cuda")
        d[torch.randperm(N, generator=g, device="cuda")[:_routed(case, N)]] = 1
        s["d"] = d
        s["O"] = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda")
    if own:                                                  # the descriptions and the workspace that a program keeps
        s.update(_handles(s))
    return s


def _routed(case, N):
    return 0 if case["density"] == 0 else max(1, round(case["density"] * N))


def _handles(s):
    from paper_2603_17484_b200 import l2a

    c = s["case"]
    p = l2a.params(c["B"], s["most_new"], s["most"], c["Hq"], c["Hkv"], c["D"], c["W"])
    h = {"l2a": l2a, "p": p,
         "cache": l2a.cache(s["K"], s["V"], s["table"], s["lengths"], k_scale=s.get("eK"), v_scale=s.get("eV"))}
    if c["kind"] == "attend":
        h["ws"] = torch.empty(l2a.l2a_cache_workspace_bytes(p, h["cache"], s["N"]), dtype=torch.uint8, device="cuda")
    return h


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend}[kind](s)
    l2a = s["l2a"]
    if kind == "append":
        l2a.l2a_cache_append(s["p"], s["cache"], s["newK"], s["newV"], s["cu"], s["N"])
        return _pool(s)
    if kind == "read":
        l2a.l2a_cache_read(s["p"], s["cache"], None, s["outK"], s["outV"])
        return {"K": s["outK"], "V": s["outV"]}
    l2a.l2a_cache_forward(s["p"], s["cache"], s["Q"], s["cu"], s["N"], s["d"], s["O"], s["ws"])
    return s["O"]


def _pool(s):
    """The pool as it is held: 8-bit floats and the exponents of their scales, or bf16."""
    return {k: s[k] for k in ("K", "V", "eK", "eV") if k in s}


# ---------------------------------------------------------------------------------------------------- plain forms
def _positions(s):
    """Sequence and position of every new token."""
    t = torch.arange(s["N"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    return b, s["lengths"][b] - s["cu"][b + 1] + t


def _plain_append(s):
    page = s["case"]["page"]
    b, pos = _positions(s)
    at, slot = s["table"][b, pos // page].long(), (pos % page).long()
    if "eK" not in s:
        s["K"][at, :, slot] = s["newK"]
        s["V"][at, :, slot] = s["newV"]
        return _pool(s)
    K, s["eK"][at, :, slot] = _quantised(s["newK"])
    V, s["eV"][at, :, slot] = _quantised(s["newV"])
    s["K"].view(torch.uint8)[at, :, slot] = K.view(torch.uint8)
    s["V"].view(torch.uint8)[at, :, slot] = V.view(torch.uint8)
    return _pool(s)


def _plain_dense(s, name):
    """[B, Hkv, keys, D] in 32 bits, zeros behind a sequence's end."""
    c = s["case"]
    at = s["table"].long().clamp(min=0)
    x = s[name][at].float()
    if "e" + name in s:
        x = x * (s["e" + name][at].int() << 23).view(torch.float32).unsqueeze(-1)
    x = x.permute(0, 2, 1, 3, 4).reshape(c["B"], c["Hkv"], -1, c["D"])[:, :, :s["most"]]
    j = torch.arange(s["most"], device="cuda")
    return torch.where((j < s["lengths"][:, None])[:, None, :, None], x, 0.0)


def _plain_read(s):
    return {name: _plain_dense(s, name).transpose(1, 2).to(torch.bfloat16).contiguous() for name in ("K", "V")}


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hkv, D, L = c["B"], c["Hq"], c["Hkv"], c["D"], s["most_new"]
    K, V = _plain_dense(s, "K"), _plain_dense(s, "V")
    b, pos = _positions(s)
    i = torch.arange(s["N"], device="cuda") - s["cu"][b]
    Q = torch.zeros((B, L, Hq, D), device="cuda")
    Q[b, i] = s["Q"].float()
    p = torch.full((B, L), -1, dtype=torch.int32, device="cuda")
    p[b, i] = pos
    Q = Q.view(B, L, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    S = (Q @ K.transpose(2, 3)).mul_(D ** -0.5).view(B, Hkv, L, Hq // Hkv, -1)
    j = torch.arange(s["most"], device="cuda", dtype=torch.int32)
    seen = (j <= p[:, :, None])[:, None, :, None, :]
    S.masked_fill_(~seen, -math.inf)
    near = (j >= p[:, :, None] - c["W"])[:, None, :, None, :]
    S.sub_(S.amax(-1, keepdim=True).clamp(min=-1e30))
    glb = S.exp()
    a = (glb.view(B, Hkv, -1, glb.shape[-1]) @ V).view(B, Hkv, L, -1, D) / glb.sum(-1, keepdim=True).clamp(min=1e-38)
    del glb
    S.masked_fill_(~near, -math.inf)
    S.sub_(S.amax(-1, keepdim=True).clamp(min=-1e30))
    loc = S.exp_()
    o = (loc.view(B, Hkv, -1, loc.shape[-1]) @ V).view(B, Hkv, L, -1, D) / loc.sum(-1, keepdim=True).clamp(min=1e-38)
    d = torch.zeros((B, L), device="cuda")
    d[b, i] = s["d"].float()
    o = o + d[:, None, :, None, None] * a
    return o.permute(0, 2, 1, 3, 4).reshape(B, L, Hq, D)[b, i].to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _decoded(codes, exponents):
    """What 8-bit codes stand for, from the bits: sign, four bits of exponent (bias 7), three of mantissa."""
    c = codes.view(torch.uint8).int()
    mant, ex, sign = c & 7, (c >> 3) & 15, 1 - 2 * (c >> 7)
    whole = torch.where(ex > 0, mant + 8, mant).double()
    return sign * whole * torch.exp2((ex.clamp(min=1) - 10 + exponents.int().unsqueeze(-1) - 127).double())


def _coded(x):
    """Rows as 8-bit floats and biased exponents of their scales, all in 64 bits: the least whole e >= -126 with
    max |x| <= 448 * 2^e, and x / 2^e rounded to four significant bits, ties to even, no finer than 2^-9."""
    x = x.double()
    top = x.abs().amax(-1)
    mant, e = torch.frexp(top / E4M3_MAX)                    # the least power of two not below: 2^(e - 1) for mant = 1/2
    e = torch.where(top > 0, e - (mant == 0.5).int(), 0).clamp(-126, 127).double()
    x = x / torch.exp2(e).unsqueeze(-1)
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step, e + 127


def _sequence(s, name, b, length, g):
    """Keys or values of KV head g of sequence b, [length, D], in 64 bits."""
    pages = s["table"][b, :-(-length // s["case"]["page"])].long()
    x = s[name][pages, g]
    x = _decoded(x, s["e" + name][pages, g]) if "e" + name in s else x.double()
    return x.reshape(-1, x.shape[-1])[:length]


def exact(case, seed):
    s = prepare(case, seed)
    length, n = _lengths(case)
    page, D, Hkv, G = case["page"], case["D"], case["Hkv"], case["Hq"] // case["Hkv"]
    if case["kind"] == "append":
        pool = {name: (x.double() if x.dtype != torch.uint8 else None) for name, x in _pool(s).items()}
        for b in range(case["B"]):
            new = range(length[b] - n[b], length[b])
            at = s["table"][b][torch.tensor([x // page for x in new], device="cuda")].long()
            slot = torch.tensor([x % page for x in new], device="cuda")
            rows = slice(sum(n[:b]), sum(n[:b + 1]))
            for name in ("K", "V"):
                new = s["new" + name][rows]
                pool[name][at, :, slot] = _coded(new)[0] if "e" + name in s else new.double()
        return pool
    if case["kind"] == "read":
        out = {name: torch.zeros((case["B"], s["most"], Hkv, D), dtype=torch.float64, device="cuda") for name in ("K", "V")}
        for b in range(case["B"]):
            for g in range(Hkv):
                out["K"][b, :length[b], g] = _sequence(s, "K", b, length[b], g)
                out["V"][b, :length[b], g] = _sequence(s, "V", b, length[b], g)
        return out
    O = torch.zeros((s["N"], case["Hq"], D), dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        rows = slice(sum(n[:b]), sum(n[:b + 1]))
        p = torch.arange(length[b] - n[b], length[b], device="cuda")[:, None]
        j = torch.arange(length[b], device="cuda")
        routed = s["d"][rows].double()
        for g in range(Hkv):
            K, V = _sequence(s, "K", b, length[b], g), _sequence(s, "V", b, length[b], g)
            for h in range(g * G, (g + 1) * G):
                w = torch.exp(s["Q"][rows, h].double() @ K.T / math.sqrt(D))
                w = w * (j <= p)
                near = w * (j >= p - case["W"])
                O[rows, h] = near @ V / near.sum(1, keepdim=True) + routed[:, None] * (w @ V / w.sum(1, keepdim=True))
    return O


# ---------------------------------------------------------------------------------------------------- work
def work(case):
    """Each key that some row sees is read once, each result written once; four operations for every visible pair of a
    query row and a key and head element, the pairs inside the window once for both attentions."""
    length, n = _lengths(case)
    N, Hq, Hkv, D, W = sum(n), case["Hq"], case["Hkv"], case["D"], case["W"]
    row = 2.0 * Hkv * (D + 1 if case["cache"] == "e4m3" else 2 * D)          # a key and its value as held
    if case["kind"] == "append":
        return {"bytes": N * (4.0 * Hkv * D + row), "flops": 0.0}
    if case["kind"] == "read":
        return {"bytes": sum(length) * row + 4.0 * case["B"] * max(length) * Hkv * D, "flops": 0.0}
    rho = _routed(case, N) / N
    keys = pairs = 0.0
    for total, new in zip(length, n):
        first = total - new
        window = total - max(0, first - W)
        some = 1 - (1 - rho) ** new                                          # the share of calls in which one is routed
        keys += window + some * (total - window)
        for p in range(first, total):
            near = min(p, W) + 1
            pairs += near + rho * (p + 1 - near)
    return {"bytes": keys * row + 4.0 * N * Hq * D, "flops": 4.0 * D * Hq * pairs}
