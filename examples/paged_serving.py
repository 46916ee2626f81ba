"""Serving one L2A layer from paged caches: prompts in chunks and single tokens of several sequences in the same steps.

The layer has projections, and so a cache, for each of its two modules.  A step of the server takes some new tokens of every
active sequence on one token axis and runs

  l2a_cache_append   keys and values of the new tokens into the pages of both caches (bf16, 8 or 4 bits)
  l2a_cache_forward  SKIP_GLOBAL: Local Attention s from the local cache
  l2a_router_logits  z = w . s + bias; a token is routed where z >= 0
  l2a_cache_forward  GLOBAL_PHASE: o = s + d a from the global cache, routed tokens only

and l2a_cache_read takes a finished sequence out of the pool.  With a bound on the tokens that a sequence keeps, a step also runs

  l2a_cache_weigh    what Global Attention of the routed tokens gives each key of the global cache, added to its weight
  l2a_cache_evict    a sequence over the bound: its first tokens, the last of a window and more, and those of the highest weights in between move to
                     other pages, a shorter cache

Run: python examples/paged_serving.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_17484_b200 import l2a  # noqa: E402


class Pool:
    """Pages of one cache.  Page numbers are shared by all caches of a server, so the server hands them out."""

    def __init__(self, n_pages, Hkv, page, D, bits, table, lengths):
        shape = (n_pages, Hkv, page, D if bits > 4 else D // 2)
        dtype = {16: torch.bfloat16, 8: torch.float8_e4m3fn, 4: torch.uint8}[bits]
        self.K, self.V = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in "KV")
        if bits == 4:
            self.K, self.V = self.K.view(torch.float4_e2m1fn_x2), self.V.view(torch.float4_e2m1fn_x2)
        scales = {16: None, 8: shape[:3], 4: (n_pages, Hkv, page * (1 + D // 16))}[bits]
        self.scales = [torch.zeros(scales, dtype=torch.uint8, device="cuda") if scales else None for _ in "KV"]
        self.handle = self.view(table, lengths)

    def view(self, table, lengths):
        """The cache of some sequences: rows of a table, and their lengths."""
        return l2a.cache(self.K, self.V, table, lengths, *self.scales)


class Layer:
    """One layer of the server: two caches, the router's weights, a workspace for the largest step."""

    def __init__(self, slots, longest, most_new, step_tokens, heads, window, page=64, bits=8, n_pages=None, bound=None):
        """bound: tokens that a sequence keeps; None: all."""
        self.Hq, self.Hkv, self.D = heads
        self.window, self.page, self.slots, self.longest = window, page, slots, longest
        per = -(-longest // page)
        n_pages = slots * per if n_pages is None else n_pages
        self.table = torch.full((slots, per), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(slots, dtype=torch.int32, device="cuda")
        self.local = Pool(n_pages, self.Hkv, page, self.D, bits, self.table, self.lengths)
        self.glob = Pool(n_pages, self.Hkv, page, self.D, bits, self.table, self.lengths)
        self.free = list(range(n_pages))[::-1]
        self.held = [0] * slots                                  # tokens of each slot
        self.most_new = most_new
        ws = l2a.l2a_cache_workspace_bytes(self._params(most_new), self.local.handle, step_tokens)
        self.ws = torch.empty(ws, dtype=torch.uint8, device="cuda")
        self.w = torch.zeros(self.Hq * self.D, device="cuda")
        self.bias = 0.0
        self.bound, self.first = bound, 4
        if bound is not None:
            self.weights = torch.zeros((n_pages, self.Hkv, page), device="cuda")
            self.weigh_ws = torch.empty(l2a.l2a_cache_weigh_workspace_bytes(self._params(most_new), self.glob.handle, step_tokens),
                                        dtype=torch.uint8, device="cuda")

    def _params(self, most_new, flags=0):
        return l2a.params(self.slots, most_new, self.longest, self.Hq, self.Hkv, self.D, self.window, flags=flags)

    def step(self, new, local, glob):
        """new: tokens of every slot in this step; local, glob: (Q, K, V) of the tokens on one axis, in slot order.  Returns (o, d)."""
        N = sum(new)
        for slot, n in enumerate(new):                           # pages for the new tokens
            have, need = -(-self.held[slot] // self.page), -(-(self.held[slot] + n) // self.page)
            if need > have:
                pages = [self.free.pop() for _ in range(need - have)]
                self.table[slot, have:need] = torch.tensor(pages, dtype=torch.int32)
            self.held[slot] += n
        self.lengths.copy_(torch.tensor(self.held, dtype=torch.int32))
        cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32).cuda()
        most = max(new)
        p = self._params(most)
        for cache, (_, K, V) in ((self.local, local), (self.glob, glob)):
            l2a.l2a_cache_append(p, cache.handle, K, V, cu, N)
        O = torch.empty((N, self.Hq, self.D), dtype=torch.bfloat16, device="cuda")
        l2a.l2a_cache_forward(self._params(most, l2a.FLAG_SKIP_GLOBAL), self.local.handle, local[0], cu, N, None, O, self.ws)
        z = torch.empty((1, N), device="cuda")
        l2a.l2a_router_logits(l2a.params(1, N, N, self.Hq, self.Hkv, self.D, self.window), O, self.w, self.bias, z)
        d = (z[0] >= 0).to(torch.uint8)
        l2a.l2a_cache_forward(self._params(most, l2a.FLAG_GLOBAL_PHASE), self.glob.handle, glob[0], cu, N, d, O, self.ws)
        if self.bound is not None:
            l2a.l2a_cache_weigh(p, self.glob.handle, glob[0], cu, N, d, self.weights, self.weigh_ws)
            for slot, n in enumerate(self.held):
                if n > self.bound:
                    self.shrink(slot)
        return O, d

    def shrink(self, slot):
        """Evicts from both caches of a slot down to three quarters of the bound (at least what Local Attention needs)."""
        n, room = self.held[slot], max(3 * self.bound // 4, self.window + self.first)
        keep = min(n, room)
        pages = [self.free.pop() for _ in range(-(-keep // self.page))]
        table = torch.tensor([pages], dtype=torch.int32, device="cuda")
        p = l2a.params(1, keep, n, self.Hq, self.Hkv, self.D, self.window)
        kept = torch.tensor([keep], dtype=torch.int32, device="cuda")
        length = torch.empty(1, dtype=torch.int32, device="cuda")
        for cache in (self.local, self.glob):                    # (the local cache goes by the same weights: only its last tokens matter)
            old = cache.view(self.table[slot:slot + 1], self.lengths[slot:slot + 1])
            ws = torch.empty(l2a.l2a_cache_evict_workspace_bytes(p, old), dtype=torch.uint8, device="cuda")
            l2a.l2a_cache_evict(p, old, self.weights, kept, self.first, self.window, cache.view(table, length), self.weights, length, None, ws)
        self.free += self.table[slot, :-(-n // self.page)].tolist()
        self.table[slot, :len(pages)] = table[0]
        self.held[slot] = keep
        self.lengths[slot] = keep

    def take_out(self, slot):
        """Dense keys and values of both caches of a slot, [tokens, Hkv, D]; its pages go back to the pool."""
        n = self.held[slot]
        p = l2a.params(1, 1, max(n, 1), self.Hq, self.Hkv, self.D, self.window)
        got = []
        for cache in (self.local, self.glob):
            one = cache.view(self.table[slot:slot + 1], self.lengths[slot:slot + 1])
            K, V = (torch.empty((1, max(n, 1), self.Hkv, self.D), dtype=torch.bfloat16, device="cuda") for _ in "KV")
            l2a.l2a_cache_read(p, one, None, K, V)
            got.append((K[0, :n], V[0, :n]))
        pages = self.table[slot, :-(-n // self.page)].tolist()
        self.free += pages
        self.held[slot] = 0
        self.lengths[slot] = 0
        return got


def serve(prompts, answer, heads=(28, 4, 128), window=512, chunk=700, bits=8, seed=0, bound=None):
    """Prompts (their lengths) start one step after the other and are taken in chunks, then `answer` single tokens each.  Returns
    the layer's outputs of every sequence, its decisions, and (Q, K, V) of both modules, all [tokens, heads, D]."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, D = heads
    total = [n + answer for n in prompts]
    page = 64
    spare = 0 if bound is None else -(-max(total) // page)       # an eviction writes a sequence's next pages before the others are free
    layer = Layer(len(prompts), max(total), chunk, chunk * len(prompts), heads, window, page=page, bits=bits, bound=bound,
                  n_pages=len(prompts) * -(-max(total) // page) + spare)
    layer.w.normal_(generator=g)
    layer.bias = -0.8 * float(layer.w.norm()) * 0.06             # about a fifth of the tokens of random inputs
    data = [[[torch.randn((n, h, D), generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)] for _ in range(2)] for n in total]
    out, dec = [[] for _ in prompts], [[] for _ in prompts]
    done, step = [0] * len(prompts), 0
    while any(done[s] < total[s] for s in range(len(prompts))):
        new = []
        for s, n in enumerate(prompts):
            left = total[s] - done[s]
            new.append(0 if step < s or left == 0 else min(chunk, n - done[s]) if done[s] < n else 1)
        if any(new):
            parts = [[torch.cat([data[s][m][i][done[s]:done[s] + new[s]] for s in range(len(prompts))]) for i in range(3)] for m in range(2)]
            O, d = layer.step(new, *parts)
            at = 0
            for s, n in enumerate(new):
                out[s].append(O[at:at + n])
                dec[s].append(d[at:at + n])
                at += n
                done[s] += n
        step += 1
    return layer, [torch.cat(x) for x in out], [torch.cat(x) for x in dec], data


def main():
    prompts, answer = [3000, 517, 1800, 64], 20
    for bits, bound in ((16, None), (8, None), (4, None), (4, 1500)):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in "ab")
        start.record()
        layer, out, dec, _ = serve(prompts, answer, bits=bits, bound=bound)
        end.record()
        torch.cuda.synchronize()
        routed = sum(int(d.sum()) for d in dec) / sum(len(d) for d in dec)
        print(f"{bits}-bit cache{f' of at most {bound} tokens a sequence' if bound else ''}: {sum(len(o) for o in out)} tokens of {len(prompts)} sequences, {100 * routed:.0f} % routed, "
              f"{start.elapsed_time(end):.1f} ms")
        K, V = layer.take_out(0)[0]
        print(f"  sequence 0 taken out: keys {tuple(K.shape)}, {len(layer.free)} pages free")


if __name__ == "__main__":
    main()
