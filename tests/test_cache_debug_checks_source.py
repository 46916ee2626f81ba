"""The index-checking build: in the kernels of the weights of cached keys and of the eviction, places that are derived from lists, plans and pieces of work are
checked before they are stored to or formed into an address."""
import re

import pytest

from tests.test_overlapped_launches import CSRC, TEXT, kernel


def function(name):
    """From the definition of a device function on."""
    common = open(f"{CSRC}/cache_common.cuh").read()
    text = common if re.search(rf"\b{name}\(", common) else TEXT
    return text[re.search(rf"__device__[^;\n]*\b{name}\(", text).start():]


@pytest.mark.parametrize("body,store,check", [
    (lambda: function("make_plan"), "p.list[at] =", r"dbg_in_range\(at < c\.n_tokens, a\.status\)"),
    (lambda: function("make_plan"), "p.blocks[q] = r", r"dbg_in_range\(q < p\.most_blocks "),
    (lambda: function("decode_keys"), "store_32(", r"dbg_in_range\(block < out\.table_stride "),
    (lambda: kernel("weigh_rows_kernel")[1], "t * a.q_t", r"dbg_in_range\(t >= 0 && t < a\.c\.n_tokens, a\.status\)"),
    (lambda: kernel("weigh_pass_kernel")[1], "p.part[at * kTileM + r] =", r"dbg_in_range\(at < p\.parts "),
    (lambda: function("add_weights"), "red.global.add", r"dbg_in_range\(key >= 0 && key % 4 == 0 && last < c\.max_keys "),
    (lambda: kernel("cache_few_add_kernel")[1], "scores +", r"dbg_in_range\(rows <= a\.score_rows "),
    (lambda: function("few_piece_e2m1"), "dst[8 * k] =", r"dbg_in_range\(score_inside\("),
    (lambda: kernel("cache_few_kernel")[1], "dst + 8) =", r"dbg_in_range\(score_inside\("),
    (lambda: kernel("cache_few_kernel")[1], "(a.part)[", r"dbg_in_range\(part_inside\("),
    (lambda: kernel("cache_few_kernel")[1], "float* slot =", r"dbg_in_range\(part_inside\("),
    (lambda: kernel("cache_move_kernel")[1], "n.K + at", r"dbg_in_range\(inside && t < a\.most "),
])
def test_checked_before_the_store(body, store, check):
    text = body()
    assert re.search(check, text[:text.index(store)]), store
