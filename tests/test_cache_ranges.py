"""Division of the key blocks of a call over the paged cache among CTAs (csrc/cache_ranges.h), compiled for the host: calls whose sums
pass 32 bits, ragged ones, groups without keys."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2603_17484_b200 import build as l2a_build
from paper_2603_17484_b200 import l2a
from tests.test_cache_host import UNSUPPORTED, cache, calls, params

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2603_17484_b200", "csrc")

# the steps of the plan, one group after the other
SOURCE = r"""
#include "cache_ranges.h"
using namespace l2a;
extern "C" void ranges(int n, const int* blocks, const uint8_t* dual, int Hkv, int ctas, int64_t* total, int64_t* base, int64_t* cost,
                       int64_t* at, int* group, int* head, int* block) {
  int64_t b = 0, c = 0;
  for (int q = 0; q < n; ++q) {
    base[q] = b;
    cost[q] = c;
    b += (int64_t)blocks[q] * Hkv;
    c += group_cost(blocks[q], dual[q], Hkv);
  }
  total[0] = b;
  total[1] = c;
  for (int x = 0; x < ctas; ++x) {
    const int64_t want = range_cost(x, ctas, c);
    int q = n - 1;
    while (cost[q] > want || blocks[q] == 0) --q;
    const RangePlace p = range_place(want - cost[q], blocks[q], dual[q]);
    group[x] = q; head[x] = p.head; block[x] = p.block;
    at[x] = range_first(base[q], p, blocks[q]);
  }
}
"""


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    d = tmp_path_factory.mktemp("ranges")
    src = d / "ranges.cpp"
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-fPIC",
                           "-shared", "-I", CSRC, "-o", str(d / "ranges.so"), str(src)])
    lib = ctypes.CDLL(str(d / "ranges.so"))

    def call(blocks, dual, Hkv, ctas):
        n = len(blocks)
        blocks, dual = np.asarray(blocks, np.int32), np.asarray(dual, np.uint8)
        total, base, cost, at = (np.zeros(k, np.int64) for k in (2, n, n, ctas))
        place = [np.zeros(ctas, np.int32) for _ in range(3)]
        lib.ranges(n, *(x.ctypes.data_as(ctypes.c_void_p) for x in (blocks, dual)), Hkv, ctas,
                   *(x.ctypes.data_as(ctypes.c_void_p) for x in (total, base, cost, at, *place)))
        return total, base, at, place
    return call


def verify(ranges, blocks, dual, Hkv, ctas=148):
    (n_blocks, cost), base, at, (group, head, block) = ranges(blocks, dual, Hkv, ctas)
    want = sum(int(b) for b in blocks) * Hkv
    assert n_blocks == want
    assert cost == sum((int(b) * (5 if two else 8) + 40) * Hkv for b, two in zip(blocks, dual) if b)
    assert at[0] == 0 and (np.diff(at) >= 0).all() and at[-1] < want
    for x in range(ctas):
        q = group[x]
        assert 0 <= head[x] < Hkv and 0 <= block[x] < blocks[q]
        assert at[x] == base[q] + int(head[x]) * int(blocks[q]) + block[x]
    # even: no range has more than its share of the costs and what an item's own cost lets it take
    sizes = np.diff(np.append(at, want))
    assert sizes.max() <= cost / ctas / 5 + 1 + 40
    return want, cost


def test_a_million_routed_tokens(ranges):
    """32 query heads on 8, every one of 2^20 tokens routed: key blocks of the prefixes, and of windows of 4096."""
    groups = (1 << 20) * 4 // 256
    first = np.arange(groups) * 64                               # first token of a group
    loc = (first + 63) // 128 - np.maximum(first - 4096, 0) // 128 + 1
    out = np.maximum(first + 63 - 4097, -1) // 128 + 1
    blocks = np.concatenate([loc, out])
    want, cost = verify(ranges, blocks, np.zeros(len(blocks)), 8)
    assert cost > 1 << 32 and want > 1 << 28


def test_more_blocks_than_32_bits(ranges):
    """131072 items of 2.6 million keys."""
    want, _ = verify(ranges, np.full(1 << 14, 20500), np.zeros(1 << 14), 8)
    assert want > 1 << 31


def test_ragged_groups(ranges):
    r = np.random.default_rng(3)
    for _ in range(50):
        n = int(r.integers(1, 60))
        blocks = (2 ** r.uniform(0, 10, n)).astype(int) * (r.random(n) < 0.7)
        blocks[r.integers(n)] = 1
        dual = r.random(n) < 0.3
        Hkv = int(r.integers(1, 9))
        verify(ranges, blocks, dual, Hkv, min(148, int(blocks.sum()) * Hkv))


def test_calls_whose_blocks_cannot_be_counted_are_refused():
    """2^23 rows of one KV head over 2^31 - 1 keys: 2 (2^15 + 1) groups of 2^24 blocks each are past 2^38; half the keys are not."""
    l2a_build.build_lib()
    c = cache(table_stride=1 << 24, page_size=128)
    n = 1 << 21
    big, half = (params(B=1, Lq=n, Lk=Lk, Hq=4, Hkv=1) for Lk in ((1 << 31) - 1, (1 << 28) - 1))
    assert calls(big, c, n=n)[2] == UNSUPPORTED
    assert l2a.l2a_cache_workspace_bytes(half, c, n) > 0
    with pytest.raises(l2a.L2AError):
        l2a.l2a_cache_workspace_bytes(big, c, n)


def test_sequences_whose_tiles_cannot_be_counted_are_refused():
    """One sequence of few rows over 2^31 - 1 keys: 2^25 tiles, which 296 ranges round up past 2^31."""
    c = cache(table_stride=1 << 24, page_size=128)
    assert calls(params(B=1, Lq=1, Lk=(1 << 31) - 1, Hq=1, Hkv=1), c, n=1)[2] == UNSUPPORTED
    assert l2a.l2a_cache_workspace_bytes(params(B=1, Lq=1, Lk=1 << 28, Hq=1, Hkv=1), c, 1) > 0
