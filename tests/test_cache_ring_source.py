"""4-bit caches, few rows: the warps of a CTA take the tiles of its ring in turn and wait on every other one alone.  A wait tells a phase of a stage from the
next by its parity only, so that the ring must have a whole number of turns.  The ring in numbers, and that the kernel's build insists on it."""
import re

import pytest

from tests.test_overlapped_launches import TEXT


def first_early_wait(stages, turns, tiles=60):
    """The first tile whose wait a warp can pass before the tile has landed, None if there is none.  Phase n of a stage is its n-th tile; a wait for
    its parity passes as soon as the phase ahead of it is the last one complete or the phase itself is.  The phase ahead is certain to be complete
    only if the warp has waited for it itself (copies land in any order)."""
    for t in range(stages, tiles):
        if (t - stages) % turns != t % turns:
            return t
    return None


@pytest.mark.parametrize("stages,turns,ok", [(6, 2, True), (4, 2, True), (5, 2, False), (6, 4, False), (4, 4, True), (5, 1, True)])
def test_turns_and_stages(stages, turns, ok):
    assert (first_early_wait(stages, turns) is None) == ok == (stages % turns == 0)


def test_the_build_insists_on_whole_turns():
    assert re.search(r"kTurns = kKind == L2A_CACHE_E2M1 \? kE2m1Steps : 1", TEXT)
    assert re.search(r"static_assert\(kStages >= 2 && kStages % kTurns == 0", TEXT)
    body = TEXT[TEXT.index("bool few_piece_e2m1("):]
    assert re.search(r"if \(t % kSteps != warp / kWarps\) continue;", body)
