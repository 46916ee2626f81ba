"""Serving one L2A layer from paged caches: prompts in chunks and single tokens of several sequences in the same steps.

The layer has projections, and so a cache, for each of its two modules.  A step of the server takes some new tokens of every
active sequence on one token axis and runs

  l2a_cache_append   keys and values of the new tokens into the pages of both caches (8 bits or bf16)
  l2a_cache_forward  SKIP_GLOBAL: Local Attention s from the local cache
  l2a_router_logits  z = w . s + bias; a token is routed where z >= 0
  l2a_cache_forward  GLOBAL_PHASE: o = s + d a from the global cache, routed tokens only

and l2a_cache_read takes a finished sequence out of the pool.  Run: python examples/paged_serving.py
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
        shape = (n_pages, Hkv, page, D)
        dtype = torch.float8_e4m3fn if bits == 8 else torch.bfloat16
        self.K, self.V = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in "KV")
        ks, vs = ((torch.zeros(shape[:3], dtype=torch.uint8, device="cuda") for _ in "KV") if bits == 8 else (None, None))
        self.handle = l2a.cache(self.K, self.V, table, lengths, k_scale=ks, v_scale=vs)


class Layer:
    """One layer of the server: two caches, the router's weights, a workspace for the largest step."""

    def __init__(self, slots, longest, most_new, step_tokens, heads, window, page=64, bits=8, n_pages=None):
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
        return O, d

    def take_out(self, slot):
        """Dense keys and values of both caches of a slot, [tokens, Hkv, D]; its pages go back to the pool."""
        n = self.held[slot]
        p = l2a.params(1, 1, max(n, 1), self.Hq, self.Hkv, self.D, self.window)
        got = []
        for cache in (self.local, self.glob):
            h = cache.handle
            one = l2a.cache(cache.K, cache.V, self.table[slot:slot + 1], self.lengths[slot:slot + 1],
                            k_scale=h.tensors[2], v_scale=h.tensors[3])
            K, V = (torch.empty((1, max(n, 1), self.Hkv, self.D), dtype=torch.bfloat16, device="cuda") for _ in "KV")
            l2a.l2a_cache_read(p, one, None, K, V)
            got.append((K[0, :n], V[0, :n]))
        pages = self.table[slot, :-(-n // self.page)].tolist()
        self.free += pages
        self.held[slot] = 0
        self.lengths[slot] = 0
        return got


def serve(prompts, answer, heads=(28, 4, 128), window=512, chunk=700, bits=8, seed=0):
    """Prompts (their lengths) start one step after the other and are taken in chunks, then `answer` single tokens each.  Returns
    the layer's outputs of every sequence, its decisions, and (Q, K, V) of both modules, all [tokens, heads, D]."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, D = heads
    total = [n + answer for n in prompts]
    layer = Layer(len(prompts), max(total), chunk, chunk * len(prompts), heads, window, bits=bits)
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
    for bits in (16, 8):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in "ab")
        start.record()
        layer, out, dec, _ = serve(prompts, answer, bits=bits)
        end.record()
        torch.cuda.synchronize()
        routed = sum(int(d.sum()) for d in dec) / sum(len(d) for d in dec)
        print(f"{bits}-bit cache: {sum(len(o) for o in out)} tokens of {len(prompts)} sequences, {100 * routed:.0f} % routed, "
              f"{start.elapsed_time(end):.1f} ms")
        K, V = layer.take_out(0)[0]
        print(f"  sequence 0 taken out: keys {tuple(K.shape)}, {len(layer.free)} pages free")


if __name__ == "__main__":
    main()
